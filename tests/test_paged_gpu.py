"""Attention over paged caches against the definition in 64 bits: types, head layouts, page sizes, ragged
batches, lengths from nothing to cut over many work-groups, hidden memory, streams and captured graphs."""
import numpy as np
import pytest
import torch

from paged_util import Paged, compare
from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu

TYPES = [("f32", "f32"), ("f32", "e4m3"), ("bf16", "bf16"), ("bf16", "e4m3")]


def bits(t):
    return t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n,lens,H_q,H_kv,D,page", [
    ([1], [1], 4, 1, 64, 16),
    ([1], [300], 4, 1, 64, 16),
    ([1, 1, 1], [17, 64, 65], 28, 4, 128, 16),
    ([1] * 9, [1, 700, 63, 128, 1000, 2, 33, 511, 64], 28, 4, 128, 64),
    ([2, 9, 1, 4], [5, 777, 130, 1200], 32, 8, 64, 16),
    ([5], [2000], 7, 1, 128, 256),
    ([32], [1500], 28, 4, 128, 64),
    ([70], [70], 28, 4, 128, 32),
    ([33, 0, 129], [33, 40, 1029], 16, 2, 128, 128),
    ([150], [400], 8, 8, 64, 1024),
    ([3, 1], [900, 333], 24, 24, 128, 32),
    ([2, 3], [100, 600], 160, 4, 64, 16),
])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_against_64_bits(dtype, cache, n, lens, H_q, H_kv, D, page, causal):
    c = Paged(n, lens, H_q, H_kv, D, page, dtype, cache, seed=len(n) + lens[-1])
    out, lse = c.attn(causal=causal)
    torch.cuda.synchronize()
    compare(dtype, out, lse, c.reference(causal), f"{dtype}/{cache}")


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n,lens,H_q,H_kv,D", [
    ([1], [9000], 28, 4, 128),              # one axis cut over all work-groups
    ([1, 1, 1, 1, 1], [5000, 3, 800, 1, 2500], 7, 1, 128),
    ([40, 3], [4100, 6000], 8, 4, 64),
    ([300], [3000], 14, 2, 128),
    ([200, 1, 0, 17, 64], [200, 3000, 9, 1700, 640], 14, 2, 128),
])
def test_long_axes_cut_over_work_groups(dtype, cache, n, lens, H_q, H_kv, D):
    c = Paged(n, lens, H_q, H_kv, D, 64, dtype, cache, seed=5)
    assert pdec.query_paged_plan(pdec.paged_dims_of(c.put().dev["q"], c.dev["k_pages"], c.dev["block_table"]))["merge_pass"]
    out, lse = c.attn()
    compare(dtype, out, lse, c.reference(), f"{dtype}/{cache}")
    # tight bounds divide the work otherwise
    out, lse = c.attn(max_chunk=max(n), max_len=max(lens))
    compare(dtype, out, lse, c.reference(), f"{dtype}/{cache} tight")


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_many_sequences(dtype, cache):
    """More pairs than work-groups, most of them of a few keys, some without tokens."""
    rng = np.random.default_rng(3)
    S = 300
    n = rng.integers(0, 4, S).tolist()
    lens = [int(rng.integers(a, 40)) if rng.random() < 0.8 else int(rng.integers(200, 400)) for a in n]
    c = Paged(n, lens, 8, 4, 64, 16, dtype, cache, seed=6)
    out, lse = c.attn()
    compare(dtype, out, lse, c.reference(), f"{dtype}/{cache}")
    out, lse = c.attn(max_chunk=3, max_len=400)
    compare(dtype, out, lse, c.reference(), f"{dtype}/{cache} tight")


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("S,where", [(70, (0, 69)), (200, (3, 150)), (300, (299,)), (400, ())])
def test_a_few_chunks_among_many_single_tokens(dtype, cache, S, where):
    """Chunks of up to 600 tokens at a few places of a batch of single tokens and of sequences without any."""
    rng = np.random.default_rng(S)
    n = [int(rng.integers(0, 2)) for _ in range(S)]
    lens = [int(rng.integers(max(a, 1), 60)) for a in n]
    for k, s in enumerate(where):
        n[s], lens[s] = (600, 37)[k % 2], (600, 900)[k % 2]
    c = Paged(n, lens, 14, 2, 64, 16, dtype, cache, seed=S)
    for kw in ({}, {"max_chunk": max(n), "max_len": max(lens)}):
        out, lse = c.attn(**kw)
        compare(dtype, out, lse, c.reference(), f"{dtype}/{cache} {kw}")


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_absent_pages_and_rows_that_see_nothing(dtype, cache, causal):
    """Pages missing at the start, in the middle, everywhere; more new tokens than keys."""
    n, lens = [3, 40, 2, 7, 5], [400, 200, 90, 4, 0]
    absent = {(0, 0), (0, 3), (0, 12)} | {(1, i) for i in range(10)} | {(2, i) for i in range(6)}
    c = Paged(n, lens, 14, 2, 128, 16, dtype, cache, seed=8, absent=absent)
    out, lse = c.attn(causal=causal)
    ref = c.reference(causal)
    assert np.isneginf(ref[1]).any() and np.isfinite(ref[1]).any()
    compare(dtype, out, lse, ref, f"{dtype}/{cache}")


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("junk", [np.nan, np.inf, -3e38])
def test_hidden_memory_does_not_matter(dtype, cache, junk):
    """Free pages and rows behind a sequence's end hold NaN, infinities or the lowest values."""
    kw = dict(n=[1, 30, 4, 90], lens=[77, 130, 900, 90], H_q=14, H_kv=2, D=128, page=32, dtype=dtype, cache=cache, seed=9)
    a, b = Paged(**kw), Paged(**kw, junk=junk)
    (o1, l1), (o2, l2) = a.attn(), b.attn()
    assert torch.isfinite(o1.float()).all()
    assert torch.equal(bits(o1), bits(o2)) and torch.equal(bits(l1), bits(l2))


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("D,H_q,H_kv", [(64, 8, 4), (128, 14, 2), (128, 28, 1)])
def test_values_of_later_tokens_stay_with_those_that_see_them(dtype, cache, D, H_q, H_kv):
    """A chunk whose tokens 5, 20 and 41 have infinite or NaN values (and token 30 NaN keys): the tokens before
    them are as without, bit for bit."""
    n, lens = [60, 3], [190, 75]
    c = Paged(n, lens, H_q, H_kv, D, 16, dtype, cache, seed=10).put()
    o1, l1 = (x.clone() for x in c.attn())
    nan = float("nan")
    for tok, val in ((5, nan), (20, float("inf")), (41, -float("inf"))):
        t = lens[0] - n[0] + tok
        page, row = int(c.table[0, t // 16]), t % 16
        if cache == "e4m3":
            c.dev["v_pages"].view(torch.uint8)[page, row] = 0x7F
            c.vals["v"][page, row] = np.nan
        else:
            c.dev["v_pages"][page, row] = val
            c.vals["v"][page, row] = val
    t = lens[0] - n[0] + 30
    page, row = int(c.table[0, t // 16]), t % 16
    c.dev["k_pages"].view(torch.uint8)[page, row, :, :] = 0x7F if cache == "e4m3" else 0xFF
    o2, l2 = c.attn()
    assert torch.equal(bits(o1[:5]), bits(o2[:5])) and torch.equal(bits(l1[:30]), bits(l2[:30]))
    assert torch.equal(bits(o1[60:]), bits(o2[60:])) and torch.equal(bits(l1[60:]), bits(l2[60:]))
    o = o2.float().cpu().numpy()
    assert np.isnan(o[30:60]).all()  # they see a NaN key
    if cache == "e4m3":
        assert np.isnan(o[5:30]).all()
    else:
        assert np.isnan(o[5:20]).all()


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_rows_behind_the_last_sequence_stay(dtype, cache):
    c = Paged([3, 50], [40, 500], 14, 2, 64, 16, dtype, cache, seed=11, pad=37).put()
    out = torch.full_like(c.dev["q"], 7.0)
    lse = torch.full(out.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    c.attn(out=out, lse=lse)
    compare(dtype, out, lse, c.reference(), "padded")
    assert (out[53:] == 7).all() and (lse[53:] == 7).all()


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_calls_agree_bit_for_bit_whatever_the_workspace_holds(dtype, cache):
    c = Paged([1, 20, 200], [3000, 2000, 700], 14, 2, 128, 64, dtype, cache, seed=12).put()
    dims = pdec.paged_dims_of(c.dev["q"], c.dev["k_pages"], c.dev["block_table"])
    ws = torch.full((pdec.paged_workspace_size(dims),), 0xFF, dtype=torch.uint8, device="cuda")
    o1, l1 = c.attn(workspace=ws)
    o2, l2 = c.attn(workspace=ws)
    o3, l3 = c.attn()
    for o, l in ((o2, l2), (o3, l3)):
        assert torch.equal(bits(o1), bits(o)) and torch.equal(bits(l1), bits(l))
    o4, none = c.attn(want_lse=False)
    assert none is None and torch.equal(bits(o1), bits(o4))


@pytest.mark.parametrize("n,H_q,H_kv,D,dtype,cache,few,many", [
    (3, 8, 2, 64, "bf16", "bf16", 16, 0), (3, 12, 3, 64, "bf16", "bf16", 16, 0), (4, 14, 2, 64, "bf16", "e4m3", 32, 0),
    (4, 7, 1, 64, "bf16", "e4m3", 32, 0), (11, 8, 2, 64, "bf16", "bf16", 48, 0), (11, 12, 3, 64, "bf16", "e4m3", 48, 0),
    (11, 8, 2, 128, "bf16", "bf16", 0, 128), (9, 14, 2, 128, "bf16", "e4m3", 0, 128), (9, 21, 3, 128, "bf16", "e4m3", 0, 128),
    (16, 12, 3, 64, "bf16", "bf16", 64, 0), (16, 8, 2, 64, "bf16", "e4m3", 64, 0), (2, 14, 2, 128, "bf16", "e4m3", 16, 0),
    (4, 21, 3, 128, "bf16", "bf16", 32, 0), (17, 12, 3, 128, "bf16", "bf16", 0, 128), (31, 8, 2, 64, "bf16", "e4m3", 0, 128),
    (33, 12, 3, 64, "bf16", "bf16", 64, 256), (70, 14, 2, 128, "bf16", "e4m3", 32, 256),
    (2, 8, 2, 64, "f32", "f32", 16, 0), (40, 8, 2, 128, "f32", "e4m3", 32, 0)])
@pytest.mark.parametrize("lens", [[200], [2900], [250, 70, 130], [900, 2900, 70], [100] * 20])
def test_every_kernel_of_the_plan(n, H_q, H_kv, D, dtype, cache, few, many, lens):
    """The rows per item that a chunk gets, whole pairs and cut ones, one state or many to a pair."""
    ns = [n] + [1 + (5 * i) % n for i in range(1, len(lens))]
    c = Paged(ns, lens, H_q, H_kv, D, 32, dtype, cache, seed=n).put()
    dims = pdec.paged_dims_of(c.dev["q"], c.dev["k_pages"], c.dev["block_table"], max_chunk=n, max_len=max(lens))
    plan = pdec.query_paged_plan(dims)
    assert (plan["rows_few"], plan["rows_many"]) == (few if not many or len(lens) > 1 else 0, many)
    assert plan["merge_pass"] == (max(lens) > 256)
    out, lse = c.attn(max_chunk=n, max_len=max(lens))
    compare(dtype, out, lse, c.reference(), f"{lens}")


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("page", [64, 256])
def test_holes_under_many_rows(dtype, cache, page):
    """Pages of whole stages absent at the front, inside and at the end, under chunks with rows in every tile."""
    n, lens = [40, 300, 9], [2000, 1700, 1500]
    absent = {(0, 0), (1, 0), (1, 1), (1, 3), (1, 1600 // page), (2, 0), (2, 2)}
    c = Paged(n, lens, 14, 2, 128, page, dtype, cache, seed=21, absent=absent)
    for causal in (True, False):
        out, lse = c.attn(causal=causal)
        compare(dtype, out, lse, c.reference(causal), f"{dtype}/{cache} {page} {causal}")


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_two_calls_at_once(dtype, cache):
    """Calls under way on two streams, each with a workspace of its own, have the bits that each has alone."""
    cs = [Paged([1, 70], [1500, 2600], 14, 2, 128, 64, dtype, cache, seed=22).put(),
          Paged([5] * 6, [800, 90, 2100, 5, 64, 700], 14, 2, 128, 64, dtype, cache, seed=23).put()]
    want = [[x.clone() for x in c.attn()] for c in cs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cs], []
    for _ in range(5):
        for c, st in zip(cs, streams):
            got.append((c, c.attn(stream=st)))
    torch.cuda.synchronize()
    for c, g in got:
        for x, y in zip(want[cs.index(c)], g):
            assert torch.equal(bits(x), bits(y))


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_lengths_outside_the_contract_stay_inside_the_arrays(dtype, cache):
    """Negative, decreasing and too large lengths; sequences 0 and 4 are right, and so are their rows; rows that
    nobody has stay."""
    c = Paged([3, 2, 2, 2, 70], [300, 40, 40, 40, 400], 14, 2, 64, 16, dtype, cache, seed=24, pad=4).put()
    want, ref = [x.clone() for x in c.attn()], c.reference()
    good = list(range(3)) + list(range(9, 79))
    cu, lens = [0, 3, 5, 4, 9, 79], [300, -7, 2 ** 31 - 1, 10 ** 6, 400]
    c.dev["cu_tokens"], c.dev["seq_lens"] = c.i32(cu), c.i32(lens)
    out, lse = torch.full_like(want[0], 7.0), torch.full_like(want[1], 7.0)
    c.attn(out=out, lse=lse)
    # other lengths divide the work elsewhere, so sums associate otherwise: within the bounds, not the same bits
    compare(dtype, out[good], lse[good], [x[good] for x in ref], "rows of the right sequences")
    assert (out[79:] == 7).all() and (lse[79:] == 7).all()


def test_a_pool_beyond_32_bit_offsets():
    """Pages behind 4 GiB of a pool: 70000 pages of 64 KiB."""
    P, page, H_kv, D = 70000, 64, 4, 128
    k = torch.zeros((P, page, H_kv, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    c = Paged([2, 100], [300, 600], 28, H_kv, D, page, "bf16", seed=13).put()
    where = np.sort(np.random.default_rng(1).choice(np.arange(66000, P), c.table.max() + 1, replace=False))
    at = torch.from_numpy(where).cuda()
    used = c.dev["k_pages"].shape[0]
    at = torch.cat([at, torch.arange(used - len(where), device="cuda")])
    k[at], v[at] = c.dev["k_pages"], c.dev["v_pages"]
    table = c.i32(np.where(c.table >= 0, where[np.maximum(c.table, 0)], -1))
    out, lse = pdec.paged_attn(c.dev["q"], k, v, table, c.dev["cu_tokens"], c.dev["seq_lens"])
    compare("bf16", out, lse, c.reference(), "large pool")


def test_scale_argument():
    c = Paged([3, 20], [60, 300], 8, 2, 64, 16, "f32", seed=14)
    out, lse = c.attn(scale=0.03)
    compare("f32", out, lse, c.reference(scale=float(np.float32(0.03))), "scale")


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_on_another_stream_and_in_a_captured_graph(dtype, cache):
    """Two calls of different sizes in one graph, replayed with other work in between; each replay has the eager bits."""
    a = Paged([1] * 4, [900, 3, 77, 2000], 14, 2, 128, 64, dtype, cache, seed=15).put()
    b = Paged([130, 5], [130, 900], 14, 2, 128, 64, dtype, cache, seed=16).put()
    want = [x.clone() for c in (a, b) for x in c.attn()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [x for c in (a, b) for x in c.attn(stream=side)]
    side.synchronize()
    for x, y in zip(want, got):
        assert torch.equal(bits(x), bits(y))
    bufs = [torch.empty_like(x) for x in want]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.attn(out=bufs[0], lse=bufs[1])
        b.attn(out=bufs[2], lse=bufs[3])
    for i in range(4):
        for x in bufs:
            x.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, bufs):
            assert torch.equal(bits(x), bits(y)), i
        a.attn()  # eager work between the replays
