"""Attention over 4-bit paged caches against the definition in 64 bits: head layouts, page sizes, ragged batches,
lengths from nothing to cut over many work-groups, hidden memory, NaN blocks, streams and captured graphs."""
import numpy as np
import pytest
import torch

from paged4_util import Paged4, quantise4
from paged_util import compare
from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu

TYPES = ["f32", "bf16"]


def bits(t):
    return t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


@pytest.mark.parametrize("dtype", TYPES)
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
    ([2, 1], [513, 49], 12, 3, 64, 32),
])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_against_64_bits(dtype, n, lens, H_q, H_kv, D, page, causal):
    c = Paged4(n, lens, H_q, H_kv, D, page, dtype, seed=len(n) + lens[-1])
    out, lse = c.attn(causal=causal)
    torch.cuda.synchronize()
    compare(dtype, out, lse, c.reference(causal), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,lens,H_q,H_kv,D", [
    ([1], [9000], 28, 4, 128),              # one axis cut over all work-groups
    ([1, 1, 1, 1, 1], [5000, 3, 800, 1, 2500], 7, 1, 128),
    ([40, 3], [4100, 6000], 8, 4, 64),
    ([300], [3000], 14, 2, 128),
    ([200, 1, 0, 17, 64], [200, 3000, 9, 1700, 640], 14, 2, 128),
])
def test_long_axes_cut_over_work_groups(dtype, n, lens, H_q, H_kv, D):
    c = Paged4(n, lens, H_q, H_kv, D, 64, dtype, seed=5)
    assert pdec.query_paged_plan(pdec.paged_dims_of(c.put().dev["q"], c.dev["k_pages"], c.dev["block_table"]))["merge_pass"]
    out, lse = c.attn()
    compare(dtype, out, lse, c.reference(), dtype)
    out, lse = c.attn(max_chunk=max(n), max_len=max(lens))  # tight bounds divide the work otherwise
    compare(dtype, out, lse, c.reference(), f"{dtype} tight")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("S,where", [(70, (0, 69)), (200, (3, 150)), (300, ())])
def test_a_few_chunks_among_many_single_tokens(dtype, S, where):
    rng = np.random.default_rng(S)
    n = [int(rng.integers(0, 2)) for _ in range(S)]
    lens = [int(rng.integers(max(a, 1), 60)) for a in n]
    for k, s in enumerate(where):
        n[s], lens[s] = (600, 37)[k % 2], (600, 900)[k % 2]
    c = Paged4(n, lens, 14, 2, 64, 16, dtype, seed=S)
    for kw in ({}, {"max_chunk": max(n), "max_len": max(lens)}):
        out, lse = c.attn(**kw)
        compare(dtype, out, lse, c.reference(), f"{dtype} {kw}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,page", [(128, 16), (64, 16), (128, 32)])
def test_absent_pages_and_rows_that_see_nothing(dtype, causal, D, page):
    """Pages missing at the start, in the middle, everywhere; more new tokens than keys."""
    n, lens = [3, 40, 2, 7, 5], [400, 200, 90, 4, 0]
    absent = {(0, 0), (0, 3), (0, 12)} | {(1, i) for i in range(10)} | {(2, i) for i in range(6)}
    c = Paged4(n, lens, 14, 2, D, page, dtype, seed=8, absent={(s, i) for s, i in absent if i < -(-lens[s] // page)})
    out, lse = c.attn(causal=causal)
    ref = c.reference(causal)
    assert np.isneginf(ref[1]).any() and np.isfinite(ref[1]).any()
    compare(dtype, out, lse, ref, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
def test_hidden_memory_does_not_matter(dtype, D):
    """Free pages and rows behind a sequence's end hold any codes under scales of NaN."""
    kw = dict(n=[1, 30, 4, 90], lens=[77, 130, 900, 90], H_q=14, H_kv=2, D=D, page=32, dtype=dtype, seed=9)
    a, b = Paged4(**kw), Paged4(**kw, junk=True)
    (o1, l1), (o2, l2) = a.attn(), b.attn()
    assert torch.isfinite(o1.float()).all()
    assert torch.equal(bits(o1), bits(o2)) and torch.equal(bits(l1), bits(l2))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,H_q,H_kv,n", [(64, 8, 4, 60), (128, 14, 2, 60), (128, 28, 1, 50), (128, 4, 2, 9), (64, 4, 2, 9),
                                              (128, 10, 2, 9), (64, 14, 2, 9)])
def test_nan_blocks_of_later_tokens_stay_with_those_that_see_them(dtype, D, H_q, H_kv, n):
    """Blocks of the values of tokens 2 and 5 and of the keys of token 7 are NaN: the tokens before them are as
    without, bit for bit, and those that see a value's block have NaN in its 32 elements only."""
    lens = [190, 75]
    c = Paged4([n, 3], lens, H_q, H_kv, D, 16, dtype, seed=10).put()
    o1, l1 = (x.clone() for x in c.attn())
    first = lens[0] - n
    c.spoil("v", 0, first + 2, block=1)
    c.spoil("v", 0, first + 5, head=0, block=0)
    o2, l2 = c.attn()
    assert torch.equal(bits(o1[:2]), bits(o2[:2])) and torch.equal(bits(l1), bits(l2))
    assert torch.equal(bits(o1[n:]), bits(o2[n:]))
    nan = np.zeros((n, H_q, D), bool)
    nan[2:, :, 32:64] = True
    nan[5:, :H_q // H_kv, :32] = True
    assert np.array_equal(np.isnan(o2[:n].float().cpu().numpy()), nan)
    compare(dtype, o2, l2, c.reference(), dtype)
    c.spoil("k", 0, first + 7, head=H_kv - 1, block=0)
    o3, l3 = c.attn()
    assert torch.equal(bits(l1[:7]), bits(l3[:7])) and torch.equal(bits(o2[:7]), bits(o3[:7]))
    G = H_q // H_kv
    assert torch.isnan(l3[7:n, -G:]).all() and torch.isnan(o3[7:n, -G:].float()).all()
    assert torch.equal(bits(l1[7:, :-G]), bits(l3[7:, :-G])) and torch.equal(bits(l1[n:]), bits(l3[n:]))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_behind_the_last_sequence_stay(dtype):
    c = Paged4([3, 50], [40, 500], 14, 2, 64, 16, dtype, seed=11, pad=37).put()
    out = torch.full_like(c.dev["q"], 7.0)
    lse = torch.full(out.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    c.attn(out=out, lse=lse)
    compare(dtype, out, lse, c.reference(), "padded")
    assert (out[53:] == 7).all() and (lse[53:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_calls_agree_bit_for_bit_whatever_the_workspace_holds(dtype):
    c = Paged4([1, 20, 200], [3000, 2000, 700], 14, 2, 128, 64, dtype, seed=12).put()
    dims = pdec.paged_dims_of(c.dev["q"], c.dev["k_pages"], c.dev["block_table"])
    ws = torch.full((pdec.paged_workspace_size(dims),), 0xFF, dtype=torch.uint8, device="cuda")
    o1, l1 = c.attn(workspace=ws)
    o2, l2 = c.attn(workspace=ws)
    o3, l3 = c.attn()
    for o, l in ((o2, l2), (o3, l3)):
        assert torch.equal(bits(o1), bits(o)) and torch.equal(bits(l1), bits(l))
    o4, none = c.attn(want_lse=False)
    assert none is None and torch.equal(bits(o1), bits(o4))


@pytest.mark.parametrize("n,H_q,H_kv,D", [
    (3, 8, 2, 64), (3, 12, 3, 64), (4, 14, 2, 64), (11, 8, 2, 64), (16, 12, 3, 64), (2, 14, 2, 128), (4, 21, 3, 128),
    (8, 8, 2, 128), (9, 14, 2, 128), (5, 14, 2, 128), (12, 8, 2, 128), (9, 14, 2, 64), (31, 8, 2, 64), (33, 12, 3, 64),
    (70, 14, 2, 128)])
@pytest.mark.parametrize("lens", [[200], [2900], [250, 70, 130], [900, 2900, 70], [100] * 20])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_every_form_of_the_kernels(n, H_q, H_kv, D, lens, page):
    """The rows per item that a chunk gets, whole pairs and cut ones, one state or many to a pair."""
    ns = [n] + [1 + (5 * i) % n for i in range(1, len(lens))]
    c = Paged4(ns, lens, H_q, H_kv, D, page, "bf16", seed=n).put()
    dims = pdec.paged_dims_of(c.dev["q"], c.dev["k_pages"], c.dev["block_table"], max_chunk=n, max_len=max(lens))
    assert pdec.query_paged_plan(dims)["merge_pass"] == (max(lens) > 256)
    out, lse = c.attn(max_chunk=n, max_len=max(lens))
    compare("bf16", out, lse, c.reference(), f"{lens}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,D", [(64, 128), (256, 128), (64, 64)])
def test_holes_under_many_rows(dtype, page, D):
    n, lens = [40, 300, 9], [2000, 1700, 1500]
    absent = {(0, 0), (1, 0), (1, 1), (1, 3), (1, 1600 // page), (2, 0), (2, 2)}
    c = Paged4(n, lens, 14, 2, D, page, dtype, seed=21, absent=absent)
    for causal in (True, False):
        out, lse = c.attn(causal=causal)
        compare(dtype, out, lse, c.reference(causal), f"{dtype} {page} {causal}")


@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_outside_the_contract_stay_inside_the_arrays(dtype):
    """Negative, decreasing and too large lengths; sequences 0 and 4 are right, and so are their rows; rows that
    nobody has stay."""
    c = Paged4([3, 2, 2, 2, 70], [300, 40, 40, 40, 400], 14, 2, 64, 16, dtype, seed=24, pad=4).put()
    want, ref = [x.clone() for x in c.attn()], c.reference()
    good = list(range(3)) + list(range(9, 79))
    c.dev["cu_tokens"], c.dev["seq_lens"] = c.i32([0, 3, 5, 4, 9, 79]), c.i32([300, -7, 2 ** 31 - 1, 10 ** 6, 400])
    out, lse = torch.full_like(want[0], 7.0), torch.full_like(want[1], 7.0)
    c.attn(out=out, lse=lse)
    compare(dtype, out[good], lse[good], [x[good] for x in ref], "rows of the right sequences")
    assert (out[79:] == 7).all() and (lse[79:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_a_pool_beyond_32_bit_offsets(dtype):
    """Pages behind 4 GiB of a pool: 280000 pages of 16 KiB."""
    P, page, H_kv, D = 280000, 64, 4, 128
    k = torch.zeros((P, H_kv, page, D // 2), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    ks, vs = (torch.zeros((P, H_kv, page, D // 32), dtype=torch.uint8, device="cuda") for _ in "kv")
    c = Paged4([2, 100], [300, 600], 28, H_kv, D, page, dtype, seed=13).put()
    used = c.dev["k_pages"].shape[0]
    where = np.sort(np.random.default_rng(1).choice(np.arange(270000, P), used, replace=False))
    at = torch.from_numpy(where).cuda()
    k[at], v[at] = c.dev["k_pages"], c.dev["v_pages"]
    ks[at], vs[at] = c.dev_scales["k_scales"], c.dev_scales["v_scales"]
    table = c.i32(np.where(c.table >= 0, where[np.maximum(c.table, 0)], -1))
    out, lse = pdec.paged_attn(c.dev["q"], k, v, table, c.dev["cu_tokens"], c.dev["seq_lens"], k_scales=ks, v_scales=vs)
    compare(dtype, out, lse, c.reference(), "large pool")


@pytest.mark.parametrize("dtype", TYPES)
def test_on_other_streams_and_in_a_captured_graph(dtype):
    """Two calls of different sizes under way at once, and in one graph, replayed with other work in between; each has
    the eager bits."""
    a = Paged4([1] * 4, [900, 3, 77, 2000], 14, 2, 128, 64, dtype, seed=15).put()
    b = Paged4([130, 5], [130, 900], 14, 2, 64, 64, dtype, seed=16).put()
    want = [x.clone() for c in (a, b) for x in c.attn()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in "ab"]
    got = [x for _ in range(3) for c, st in zip((a, b), streams) for x in c.attn(stream=st)]
    torch.cuda.synchronize()
    for x, y in zip(3 * want, got):
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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 40])
def test_scales_of_every_size(dtype, n):
    """Rows whose blocks differ by powers of two from 2^-40 to 2^20, a score's scale against them."""
    c = Paged4([n, n], [700, 333], 8, 2, 128, 32, dtype, seed=30)
    rng = np.random.default_rng(2)
    for name, lo, hi in (("k", -40, 0), ("v", -40, 20)):
        x = rng.standard_normal(c.vals[name].shape) * np.repeat(2.0 ** rng.integers(lo, hi, (*c.vals[name].shape[:3], 4)), 32, -1)
        c.set(name, *quantise4(x))
    out, lse = c.attn()
    compare(dtype, out, lse, c.reference(), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("D,page", [(128, 32), (64, 64)])
@pytest.mark.parametrize("size", [-100, -64, 66, 118])
def test_values_far_from_one(dtype, n, D, page, size):
    """Values of 2^size: the small ones in all keys, the large ones in keys whose probability, some e^-136, is below
    float32's range, so that they add nothing to the others' values of about one."""
    c = Paged4([n, n], [700, 333], 8, 2, D, page, dtype, seed=33)
    rng = np.random.default_rng(4)
    k, v = (rng.standard_normal(c.vals[name].shape) for name in "kv")
    if size < 0:
        v *= 2.0 ** size
    else:
        c.q[:, :, 0] = 4
        for s, t in ((0, 5), (0, 100), (0, 640), (1, 0), (1, 200)):
            at = c.table[s, t // page], t % page
            k[at][:, 0] = -34 * D ** 0.5
            v[at][:] *= 2.0 ** size
    c.set("k", *quantise4(k))
    c.set("v", *quantise4(v))
    out, lse = c.attn()
    compare(dtype, out, lse, c.reference(), dtype)


@pytest.mark.parametrize("n,H_q,H_kv,D", [
    (3, 8, 2, 64), (4, 14, 2, 64), (16, 12, 3, 64), (2, 14, 2, 128), (8, 8, 2, 128), (31, 8, 2, 64), (70, 14, 2, 128)])
@pytest.mark.parametrize("lens", [[200], [250, 70, 130], [900, 2900, 70], [100] * 20])
@pytest.mark.parametrize("page", [16, 128])
def test_every_form_of_the_kernels_of_float32(n, H_q, H_kv, D, lens, page):
    ns = [n] + [1 + (5 * i) % n for i in range(1, len(lens))]
    c = Paged4(ns, lens, H_q, H_kv, D, page, "f32", seed=n).put()
    dims = pdec.paged_dims_of(c.dev["q"], c.dev["k_pages"], c.dev["block_table"], max_chunk=n, max_len=max(lens))
    plan = pdec.query_paged_plan(dims)
    assert plan["rows_few"] == (16 if D == 128 or n * H_q // H_kv <= 16 else 32) and plan["rows_many"] == 0
    out, lse = c.attn(max_chunk=n, max_len=max(lens))
    compare("f32", out, lse, c.reference(), f"{lens}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 40])
def test_queries_that_are_not_finite_stay_with_their_rows(dtype, n):
    """A NaN among a query's elements makes its row NaN, out and lse, and no other row of its 16."""
    c = Paged4([n, 2], [700, 300], 8, 2, 128, 64, dtype, seed=34).put()
    o1, l1 = (x.clone() for x in c.attn())
    c.dev["q"][0, 3, 77] = float("nan")
    o2, l2 = c.attn()
    assert torch.isnan(o2[0, 3].float()).all() and torch.isnan(l2[0, 3])
    o2[0, 3], l2[0, 3] = o1[0, 3], l1[0, 3]
    assert torch.equal(bits(o1), bits(o2)) and torch.equal(bits(l1), bits(l2))


@pytest.mark.parametrize("page,D", [(16, 64), (64, 64), (32, 128), (128, 128)])
def test_parts_of_more_blocks_than_are_looked_up_at_once(page, D):
    """Work-groups with runs of tens of thousands of keys: 160 sequences read one sequence's pages with one token's
    queries, and all have its result; some of its pages are absent."""
    S, L, H_kv = 160, 14000, 8
    c = Paged4([1], [L], 2 * H_kv, H_kv, D, page, "bf16", seed=31, absent=[(0, 3), (0, L // page // 2), (0, L // page - 1)]).put()
    ref = c.reference()
    q = c.dev["q"].expand(S, -1, -1).contiguous()
    table = c.dev["block_table"].expand(S, -1).contiguous()
    dims = pdec.paged_dims_of(q, c.dev["k_pages"], table, max_chunk=1, max_len=L)
    assert pdec.query_paged_plan(dims)["rows_few"] == 16
    assert S * L * H_kv / 256 > 64 * 8 * (64 if page >= 64 else 16)  # keys of a work-group; of a look-up
    out, lse = pdec.paged_attn(q, c.dev["k_pages"], c.dev["v_pages"], table, c.i32(np.arange(S + 1)), c.i32([L] * S), max_chunk=1,
                               max_len=L, **c.dev_scales)
    for s in (0, 1, 77, S - 1):
        compare("bf16", out[s:s + 1], lse[s:s + 1], ref, f"sequence {s}")
    # the others: the same keys in other divisions
    assert torch.isfinite(out.float()).all()
    spread = (lse - lse[0]).abs().max().item()
    assert spread <= 2.0 ** -15 * (abs(lse[0]).max().item() + 1)
