"""The paged attention's forms for rows of 64 (48 and 64 query rows, two heads to a work-group, other permutations in
LDS) under absent pages, junk behind a sequence's end, values of later tokens, and the scale argument in every type."""
import numpy as np
import pytest
import torch

from paged_util import Paged, compare
from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu

TYPES = [("f32", "f32"), ("f32", "e4m3"), ("bf16", "bf16"), ("bf16", "e4m3")]
# new tokens of the longest chunk, H_q, H_kv: 12 to 64 rows per kv head, the many rows' 128 and 256, odd and even heads
FORMS = [(3, 8, 2), (3, 12, 3), (7, 8, 2), (11, 8, 2), (11, 12, 3), (16, 8, 2), (15, 12, 3), (31, 8, 2), (70, 12, 3)]


def bits(t):
    return t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("n,H_q,H_kv", FORMS)
def test_holes(dtype, cache, page, n, H_q, H_kv):
    """Pages absent at the front, inside, at the end and everywhere; a sequence with more new tokens than keys."""
    ns, lens = [n, 1, n, 2, n], [1100, 700, 600, 300, max(n - 2, 1)]
    cols = [-(-t // page) for t in lens]
    absent = {(0, 0), (0, cols[0] // 2), (1, cols[1] - 1), (1, cols[1] // 3), (1, cols[1] // 3 + 1)}
    absent |= {(2, c) for c in range(cols[2]) if c % 3 != 1} | {(3, c) for c in range(cols[3])}
    absent = {(s, c) for s, c in absent if c < cols[s]}
    c = Paged(ns, lens, H_q, H_kv, 64, page, dtype, cache, seed=50 + n, absent=absent).put()
    for causal in (True, False):
        ref = c.reference(causal)
        assert np.isneginf(ref[1]).any() and np.isfinite(ref[1]).any()
        for kw in ({}, {"max_chunk": n, "max_len": max(lens)}):
            out, lse = c.attn(causal=causal, **kw)
            compare(dtype, out, lse, ref, f"{dtype}/{cache} page {page} causal {causal} {kw}")


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("junk", [np.nan, np.inf, -3e38])
@pytest.mark.parametrize("n,H_q,H_kv", FORMS)
def test_hidden_memory_does_not_matter(dtype, cache, junk, n, H_q, H_kv):
    kw = dict(n=[n, 1, n, 2], lens=[n + 3, 77, 900, 333], H_q=H_q, H_kv=H_kv, D=64, page=32, dtype=dtype, cache=cache, seed=60 + n)
    a, b = Paged(**kw), Paged(**kw, junk=junk)
    for more in ({}, {"max_chunk": n, "max_len": 900}):
        (o1, l1), (o2, l2) = a.attn(**more), b.attn(**more)
        assert torch.isfinite(o1.float()).all()
        assert torch.equal(bits(o1), bits(o2)) and torch.equal(bits(l1), bits(l2))


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n,H_q,H_kv", FORMS)
def test_values_of_later_tokens_stay_with_those_that_see_them(dtype, cache, n, H_q, H_kv):
    """The last two tokens of a chunk have NaN values, the one before them NaN keys: the tokens in front are as
    without, bit for bit, and those that see them are NaN."""
    c = Paged([n, 1], [n + 150, 75], H_q, H_kv, 64, 16, dtype, cache, seed=70 + n).put()
    more = {"max_chunk": n, "max_len": n + 150}
    o1, l1 = (x.clone() for x in c.attn(**more))
    keys, vals = (c.dev[x].view(torch.uint8) for x in ("k_pages", "v_pages"))
    at = [(int(c.table[0, t // 16]), t % 16) for t in range(150 + n - 3, 150 + n)]
    keys[at[0]] = 0x7F if cache == "e4m3" else 0xFF
    vals[at[1]] = vals[at[2]] = 0x7F if cache == "e4m3" else 0xFF
    o2, l2 = c.attn(**more)
    clean = list(range(n - 3)) + [n]
    assert torch.equal(bits(o1[clean]), bits(o2[clean])) and torch.equal(bits(l1[clean]), bits(l2[clean]))
    assert torch.isnan(o2[n - 3:n].float()).all() and torch.isnan(l2[n - 3:n]).all()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("D", [64, 128])
def test_scale_argument(dtype, cache, D):
    """In the few-row, the many-row and the float32 kernels, whole and cut."""
    for n, lens in (([3, 1], [60, 200]), ([3, 20], [2000, 300]), ([90], [900])):
        c = Paged(n, lens, 8, 2, D, 16, dtype, cache, seed=14)
        for scale in (0.03, 0.3):
            out, lse = c.attn(scale=scale, max_chunk=max(n), max_len=max(lens))
            compare(dtype, out, lse, c.reference(scale=float(np.float32(scale))), f"scale {scale}")
