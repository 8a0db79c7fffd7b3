"""PDEC_DEBUG=1 and the paged calls: valid lengths give the bits of the plain calls, invalid ones are refused before
anything is launched.  The mode is read once per process, so these run in a child process."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

RUN = r"""
import hashlib, os, sys
sys.path.insert(0, sys.argv[1]); sys.path.insert(0, sys.argv[2])
import torch
from paged_util import Paged
from paper_2607_02963_amd import pdec
debug = os.environ.get("PDEC_DEBUG") == "1"
h = hashlib.sha256()
c = Paged([1, 0, 40], [500, 3, 300], 14, 2, 64, 16, "bf16", "e4m3", seed=1).put()
k, v, sc = c.dev["k_pages"], c.dev["v_pages"], c.dev_scales
cu, table = c.dev["cu_tokens"], c.dev["block_table"]
new = torch.randn((41, 2, 64), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
after = torch.zeros(3, dtype=torch.int32, device="cuda")
before = c.i32([499, 3, 260])
pdec.paged_kv_append(new, new, k, v, table, cu, before, after, **sc)
rows = c.i32([0, 500, 503, 803])
for t in (*c.attn(), *pdec.paged_kv_read(k, v, table, c.dev["seq_lens"], rows, num_rows=803, **sc), after):
    h.update(t.float().cpu().numpy().tobytes())
print(h.hexdigest(), flush=True)
def refused(call):
    try:
        call()
    except pdec.PdecError as e:
        return e.code == pdec.PDEC_ERR_BAD_LENGTHS
    return False
if debug:
    bad_cu, bad_lens = c.i32([0, 5, 3, 41]), c.i32([500, -3, 300])
    out, kept = torch.full_like(c.dev["q"], 7.0), k.clone()
    assert refused(lambda: pdec.paged_attn(**{**c.dev, "cu_tokens": bad_cu}, **sc, out=out))
    assert refused(lambda: pdec.paged_attn(**{**c.dev, "seq_lens": bad_lens}, **sc, out=out))
    assert refused(lambda: c.attn(max_chunk=39, out=out))
    assert refused(lambda: pdec.paged_kv_append(new, new, k, v, table, bad_cu, before, after, **sc))
    assert refused(lambda: pdec.paged_kv_append(new, new, k, v, table, cu, bad_lens, after, **sc))
    assert refused(lambda: pdec.paged_kv_read(k, v, table, c.dev["seq_lens"], rows, num_rows=802, **sc))
    torch.cuda.synchronize()
    assert (out == 7).all() and torch.equal(kept.view(torch.uint8), k.view(torch.uint8))
"""


def _run(debug):
    env = {k: v for k, v in os.environ.items() if k != "PDEC_DEBUG"}
    if debug:
        env["PDEC_DEBUG"] = "1"
    r = subprocess.run([sys.executable, "-c", RUN, ROOT, os.path.join(ROOT, "tests")], capture_output=True, text=True,
                       env=env, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout.split()


def test_debug_mode_checks_the_lengths_and_changes_nothing():
    assert _run(True) == _run(False)
