"""PDEC_DEBUG=1 and the append with rotary positions, over a 4-bit cache: valid lengths give the bits of the plain call,
invalid ones are refused before anything is launched.  The mode is read once per process: a child process."""
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
from paged4_util import Paged4
from paper_2607_02963_amd import pdec
h = hashlib.sha256()
c = Paged4([1, 0, 40], [500, 3, 300], 14, 2, 64, 16, "bf16", seed=1).put()
k, v, sc = c.dev["k_pages"], c.dev["v_pages"], c.dev_scales
cu, table = c.dev["cu_tokens"], c.dev["block_table"]
x = torch.randn((41, 18, 64), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
after, before, s = c.i32([0, 0, 0]), c.i32([499, 3, 260]), pdec.rope_spec(64)
call = lambda cu, lens: pdec.paged_rope_kv_append(x[:, :14], x[:, 14:16], x[:, 16:], k, v, table, cu, lens, after, s, **sc)
for t in (call(cu, before), after, k, v, sc["k_scales"], *c.attn()):
    h.update(t.float().cpu().numpy().tobytes())
print(h.hexdigest(), flush=True)
if os.environ.get("PDEC_DEBUG") == "1":
    kept = k.clone()
    for bad in ((c.i32([0, 5, 3, 41]), before), (cu, c.i32([499, -3, 260])), (c.i32([0, 1, 1, 42]), before)):
        try:
            call(*bad)
        except pdec.PdecError as e:
            assert e.code == pdec.PDEC_ERR_BAD_LENGTHS
        else:
            raise SystemExit("not refused")
    torch.cuda.synchronize()
    assert torch.equal(kept, k)
"""


def _run(debug):
    env = {k: v for k, v in os.environ.items() if k != "PDEC_DEBUG"}
    if debug:
        env["PDEC_DEBUG"] = "1"
    r = subprocess.run([sys.executable, "-c", RUN, ROOT, os.path.join(ROOT, "tests")], capture_output=True, text=True, env=env,
                       timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout.split()


def test_debug_mode_checks_the_lengths_and_changes_nothing():
    assert _run(True) == _run(False)
