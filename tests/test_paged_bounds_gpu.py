"""A bound of the paged calls given as a tensor that a serving loop updates in place."""
import pytest
import torch

from paged_util import Paged, compare
from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu


def test_a_bound_updated_in_place_bounds_the_next_call():
    """One token more in every call over the same tensors' shapes; the bound as a CPU tensor that grows with it."""
    most, before = torch.tensor(0), torch.zeros(1, dtype=torch.int32, device="cuda")
    for length in (300, 1100):
        c = Paged([1], [length], 8, 2, 64, 16, "bf16", seed=40, cols=80, extra=80 - -(-length // 16)).put()
        most += length - int(most)
        out, lse = c.attn(max_chunk=1, max_len=most)
        compare("bf16", out, lse, c.reference(), f"{length} keys")
    new = torch.ones((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    k, v = torch.zeros_like(c.dev["k_pages"]), torch.zeros_like(c.dev["v_pages"])
    after, fits = torch.zeros_like(before), torch.tensor(1)
    for want in (1, 2):
        pdec.paged_kv_append(new, new, k, v, c.dev["block_table"], c.dev["cu_tokens"], before, after, max_len=fits)
        assert after.tolist() == [want]
        before, after = after, before
        fits += 1
