"""Writing to paged caches, reading them back, joining attention results, and the run of them together."""
import numpy as np
import pytest
import torch

from paged_util import DTYPES, HALF_STEP, Paged, bounds, compare, e4m3_values, quantise
from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu


def bits(t):
    return t.contiguous().view({4: torch.int32, 2: torch.int16, 1: torch.uint8}[t.element_size()])


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


def new_rows(T, H_kv, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((T, H_kv, D), generator=g).mul(0.7).to(DTYPES[dtype])


CASES = [  # n, keys before, H_kv, D, page
    ([1], [0], 1, 64, 16),
    ([1, 1, 1], [0, 63, 64], 4, 128, 64),
    ([5, 0, 33, 1], [11, 7, 100, 0], 2, 128, 16),
    ([300], [17], 8, 64, 128),
    ([70, 130], [1, 30], 3, 128, 32),
    ([0, 2], [5, 1023], 24, 64, 1024),
    ([1030, 0, 1, 2, 0, 0, 1015], [7, 3, 63, 127, 0, 9, 0], 4, 128, 64),  # four tokens to a wave
    ([3, 2100], [900, 5], 10, 64, 16),
]


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("f32", "e4m3"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("n,before,H_kv,D,page", CASES)
def test_append_writes_the_rows_and_nothing_else(dtype, cache, n, before, H_kv, D, page):
    lens = [a + b for a, b in zip(n, before)]
    c = Paged(n, lens, H_kv, H_kv, D, page, dtype, cache, seed=20, pad=3).put()
    k_new, v_new = new_rows(c.T, H_kv, D, dtype, 1), new_rows(c.T, H_kv, D, dtype, 2)
    out_lens = torch.full((len(n),), -7, dtype=torch.int32, device="cuda")
    lens_in = i32(before)
    want = {x: bits(c.dev[x + "_pages"]).cpu().numpy().copy() for x in "kv"}
    want_sc = {x: c.scales[x].copy() for x in "kv"} if cache == "e4m3" else None
    for x, new in (("k", k_new), ("v", v_new)):
        q = quantise(new.float().numpy()) if cache == "e4m3" else None
        for s in range(len(n)):
            for i in range(n[s]):
                t, row = before[s] + i, int(c.cu[s]) + i
                p, r = c.table[s, t // page], t % page
                if cache == "e4m3":
                    want[x][p, r] = q[0][row]
                    want_sc[x][p, :, r] = q[1][row]
                else:
                    want[x][p, r] = bits(new[row]).numpy()
    pdec.paged_kv_append(k_new.cuda(), v_new.cuda(), c.dev["k_pages"], c.dev["v_pages"], c.dev["block_table"],
                         c.dev["cu_tokens"], lens_in, out_lens, **c.dev_scales)
    assert out_lens.tolist() == lens and lens_in.tolist() == before
    for x in "kv":
        assert np.array_equal(bits(c.dev[x + "_pages"]).cpu().numpy(), want[x])
        if cache == "e4m3":
            assert np.array_equal(c.dev_scales[x + "_scales"].cpu().numpy(), want_sc[x])


def test_append_leaves_what_does_not_fit_and_drops_rows_without_a_page():
    """Sequence 0 is one row short, 1 has a bad length, 2 misses the page of its third row, 3 fits exactly."""
    page, H_kv, D = 16, 2, 64
    k = torch.zeros((8, page, H_kv, D), device="cuda")
    v = torch.zeros_like(k)
    table = i32([[0, 1], [2, 3], [4, -1], [5, 6]])
    T = 5 + 2 + 4 + 3
    new = torch.ones((T, H_kv, D), device="cuda")
    lens_out = torch.zeros(4, dtype=torch.int32, device="cuda")
    pdec.paged_kv_append(new, 2 * new, k, v, table, i32([0, 5, 7, 11, 14]), i32([28, -3, 14, 29]), lens_out)
    assert lens_out.tolist() == [28, -3, 18, 32]
    want = torch.zeros(8, page)
    want[4, 14:] = 1
    want[6, 13:] = 1
    assert torch.equal(k[:, :, 0, 0].cpu(), want) and torch.equal(v[:, :, 1, 5].cpu(), 2 * want)
    lens_out.zero_()
    pdec.paged_kv_append(new, new, k, v, table, i32([0, 5, 7, 11, 14]), i32([0, 0, 0, 0]), lens_out, max_len=4)
    assert lens_out.tolist() == [0, 2, 4, 3]


def test_cache_calls_of_a_batch_padded_with_empty_sequences():
    """3000 sequences, tokens in the first, one in the middle and the last, rows behind them all."""
    S, T = 3000, 2600
    n, lens = np.zeros(S, int), np.zeros(S, int)
    n[0], n[1700], n[-1] = 1501, 402, 600
    lens[1700] = 11
    cu, cols = np.concatenate([[0], np.cumsum(n)]), 100
    table = np.full((S, cols), -1)
    pages = iter(np.random.default_rng(3).permutation(400))
    for s in (0, 1700, S - 1):
        table[s, :-(-(n[s] + lens[s]) // 16)] = [next(pages) for _ in range(-(-(n[s] + lens[s]) // 16))]
    k = torch.zeros((400, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    new = new_rows(T, 1, 64, "bf16", 5).cuda()
    after = torch.zeros(S, dtype=torch.int32, device="cuda")
    pdec.paged_kv_append(new, -new, k, v, i32(table), i32(cu), i32(lens), after)
    assert after.tolist() == (lens + n).tolist()
    rows = np.concatenate([[0], np.cumsum(lens + n)])
    out = [torch.full((T + 20, 1, 64), 3.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    pdec.paged_kv_read(k, v, i32(table), after, i32(rows), k_out=out[0], v_out=out[1])
    want = torch.cat([new[:1501], torch.zeros_like(new[:11]), new[1501:2503]])
    assert torch.equal(out[0][:2514], want) and torch.equal(out[1][:2514], torch.where(want == 0, want, -want))
    assert (out[0][2514:] == 3).all() and (out[1][2514:] == 3).all()


def test_append_counts_of_more_sequences_than_tokens():
    S, T = 333, 2
    cu = np.minimum(np.arange(S + 1) // 150, T)
    lens = np.arange(S) % 7
    k = torch.zeros((S, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    new = torch.ones((T, 1, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros(S, dtype=torch.int32, device="cuda")
    pdec.paged_kv_append(new, new, k, k.clone(), i32(np.arange(S)[:, None]), i32(cu), i32(lens), out)
    assert out.tolist() == (lens + np.diff(cu)).tolist()
    where = torch.nonzero(k[:, :, 0, 0]).tolist()
    assert where == [[int(s), int(lens[s])] for s in np.nonzero(np.diff(cu))[0]]


@pytest.mark.parametrize("S", [65, 500, 5000])
def test_append_and_read_of_many_sequences(S):
    """Every token finds its sequence among many, some without tokens."""
    rng = np.random.default_rng(S)
    n = rng.integers(0, 4, S)
    n[:3], n[-2:] = 0, 0
    cu = np.concatenate([[0], np.cumsum(n)])
    T = int(cu[-1])
    before = rng.integers(0, 12, S)
    k = torch.zeros((S, 16, 1, 64), device="cuda")
    v = torch.zeros_like(k)
    new = torch.arange(1, T + 1, dtype=torch.float32).view(T, 1, 1).expand(T, 1, 64).contiguous().cuda()
    table, lens = i32(rng.permutation(S)[:, None]), torch.zeros(S, dtype=torch.int32, device="cuda")
    pdec.paged_kv_append(new, -new, k, v, table, i32(cu), i32(before), lens)
    assert lens.tolist() == (before + n).tolist()
    want = torch.zeros(S, 16)
    tab = table[:, 0].tolist()
    for s in range(S):
        for i in range(n[s]):
            want[tab[s], before[s] + i] = cu[s] + i + 1
    assert torch.equal(k[:, :, 0, 7].cpu(), want) and torch.equal(v[:, :, 0, 63].cpu(), -want)
    rows = np.concatenate([[0], np.cumsum(before + n)])
    kd, vd = pdec.paged_kv_read(k, v, table, lens, i32(rows), num_rows=int(rows[-1]))
    flat = np.concatenate([want[tab[s], :before[s] + n[s]].numpy() for s in range(S)])
    assert np.array_equal(kd[:, 0, 3].cpu().numpy(), flat) and np.array_equal(vd[:, 0, 3].cpu().numpy(), -flat)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_quantisation_of_hard_rows(dtype, D):
    """Ties, every binade of a row, subnormal and largest values, zeros, infinities and NaN, exact powers."""
    tiny = 2.0 ** -149 if dtype == "f32" else 2.0 ** -133
    rows = [np.zeros(D), np.full(D, 448.0), np.full(D, 448.0) * 2.0 ** 119, np.full(D, 449.0), np.full(D, 1.75),
            np.full(D, 1.7578125), np.full(D, tiny), np.linspace(-1, 1, D) * 2.0 ** -126, np.full(D, -3.3e38),
            448.0 * 2.0 ** -np.arange(D), np.where(np.arange(D) % 5 == 0, np.inf, 1.5),
            np.where(np.arange(D) % 7 == 0, np.nan, -np.arange(D) * 1.0), np.full(D, -np.inf), np.full(D, np.nan),
            -np.zeros(D)]
    mids = (e4m3_values(np.arange(126)) + e4m3_values(np.arange(1, 127))) / 2  # between neighbours: ties
    for sign in (1, -1):
        for part in np.array_split(mids, 4):
            r = np.zeros(D)
            r[:len(part)], r[-1] = sign * part, 448.0
            rows += [r, r * 2.0 ** -20]
    rng = np.random.default_rng(0)
    rows += list(rng.standard_normal((200, D)) * 2.0 ** rng.uniform(-100, 100, (200, 1)))
    x = torch.tensor(np.array(rows), dtype=torch.float32).to(DTYPES[dtype])
    T = len(rows)
    want, byte = quantise(x.float().numpy())
    k = torch.zeros(((T + 15) // 16, 16, 1, D), dtype=torch.float8_e4m3fn, device="cuda")
    v = torch.zeros_like(k)
    ks, vs = (torch.zeros((k.shape[0], 1, 16), dtype=torch.uint8, device="cuda") for _ in "kv")
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    new = x.view(T, 1, D).cuda()
    pdec.paged_kv_append(new, new.neg(), k, v, i32(np.arange(k.shape[0])[None]), i32([0, T]), i32([0]), lens,
                         k_scales=ks, v_scales=vs)
    got = k.view(torch.uint8).view(-1, D)[:T].cpu().numpy()
    assert np.array_equal(ks.view(-1)[:T].cpu().numpy(), byte) and np.array_equal(vs.cpu().numpy(), ks.cpu().numpy())
    nan = (want & 127) == 127
    assert np.array_equal((got & 127) == 127, nan) and np.array_equal(got[~nan], want[~nan])
    gv = v.view(torch.uint8).view(-1, D)[:T].cpu().numpy()
    assert np.array_equal(gv[~nan], want[~nan] ^ 128)
    # a rounding is off by half a step at most: 2^-4 of the value, or 2^-10 of the scale
    fin = np.isfinite(x.float().numpy()).all(1) & (np.abs(x.float().numpy()).max(1) <= 448 * 2.0 ** 119)
    val = e4m3_values(got) * 2.0 ** (byte.astype(float) - 127)[:, None]
    xx = x.double().numpy()
    err = np.abs(val[fin] - xx[fin])
    assert (err <= np.maximum(2.0 ** -4 * np.abs(xx[fin]), 2.0 ** (byte[fin].astype(float) - 137)[:, None])).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_reading_back_every_byte(dtype):
    """All 256 e4m3 patterns under every scale byte that the append writes, and 0."""
    D, page = 64, 64
    table = np.arange(16)[None]
    byte = np.array([0, 1, 2, 60, 127, 128, 200, 246] + list(range(3, 251)), np.uint8)[:, None].repeat(4, 1)  # [256, 4]
    data = np.tile(np.arange(256, dtype=np.uint8).reshape(4, 64), (256, 1, 1))  # token, head, D
    k = torch.from_numpy(data.reshape(4, page, 4, D)).view(torch.float8_e4m3fn).cuda()
    sc = torch.from_numpy(np.ascontiguousarray(byte.reshape(4, page, 4).transpose(0, 2, 1))).cuda()
    ko, vo = pdec.paged_kv_read(k, k, i32(table[:, :4]), i32([256]), i32([0, 256]), num_rows=256, dtype=DTYPES[dtype],
                                k_scales=sc, v_scales=sc)
    scale = np.where(byte == 0, 0.0, 2.0 ** (byte.astype(np.float64) - 127))
    want = torch.from_numpy(e4m3_values(data) * scale[..., None]).to(torch.float32).to(DTYPES[dtype])
    for got in (ko.cpu(), vo.cpu()):
        nan = torch.isnan(want)
        assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("f32", "e4m3"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("lens,rows,H_kv,D,page", [
    ([1], [1], 1, 64, 16),
    ([100, 0, 33], [100, 0, 33], 4, 128, 16),
    ([100, 7, 64], [40, 20, 64], 2, 128, 64),     # fewer rows than keys, more rows than keys
    ([1000], [1000], 24, 64, 256),
    ([1, 2, 3, 4, 5, 6, 7], [1, 2, 3, 4, 5, 6, 7], 8, 128, 32),
])
def test_read_gives_the_rows_and_zeros(dtype, cache, lens, rows, H_kv, D, page):
    absent = {(0, 1)} if lens[0] > 2 * page else ()
    c = Paged([0] * len(lens), lens, H_kv, H_kv, D, page, dtype, cache, seed=21, absent=absent, pad=1).put()
    cu = np.concatenate([[0], np.cumsum(rows)])
    R = int(cu[-1]) + 5
    ko, vo = (torch.full((R, H_kv, D), 9.0, dtype=DTYPES[dtype], device="cuda") for _ in "kv")
    pdec.paged_kv_read(c.dev["k_pages"], c.dev["v_pages"], c.dev["block_table"], c.dev["seq_lens"], i32(cu), k_out=ko,
                       v_out=vo, **c.dev_scales)
    for x, got in (("k", ko), ("v", vo)):
        want = np.full((R, H_kv, D), 9.0)
        for s in range(len(lens)):
            rowsof, ok = c.keys(x, s)
            m = min(rows[s], lens[s])
            want[cu[s]:cu[s + 1]] = 0
            want[cu[s]:cu[s] + m] = np.where(ok[:m, None, None], rowsof[:m], 0)
        assert np.array_equal(got.double().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,D", [((1,), 64), ((7, 28), 128), ((3, 5, 11), 64), ((1000, 28), 128)])
def test_merge_against_64_bits(dtype, rows, D):
    g = torch.Generator().manual_seed(3)
    oa, ob = (torch.randn((*rows, D), generator=g).to(DTYPES[dtype]) for _ in "ab")
    la, lb = (torch.randn(rows, generator=g) * 30 for _ in "ab")
    out, lse = pdec.merge_states(oa.cuda(), la.cuda(), ob.cuda(), lb.cuda())
    a, b = la.double(), lb.double()
    share = torch.sigmoid(a - b)[..., None]
    want = share * oa.double() + (1 - share) * ob.double()
    # la - lb is rounded (2^-24 of at most 200), exp, the sum, the quotient and the products a few half steps each;
    # then out is rounded
    size = share * oa.double().abs() + (1 - share) * ob.double().abs()
    tol = size * (200 + 16) * 2.0 ** -24 + want.abs() * HALF_STEP[dtype] * 1.01 + 1e-37
    assert ((out.cpu().double() - want).abs() <= tol).all()
    want = torch.logaddexp(a, b)
    assert ((lse.cpu().double() - want).abs() <= 2.0 ** -21 + want.abs() * 2.0 ** -23).all()
    # in place, either side
    for side in (0, 1):
        o, l = [oa.cuda(), ob.cuda()], [la.cuda(), lb.cuda()]
        pdec.merge_states(o[0], l[0], o[1], l[1], out=o[side], lse=l[1 - side])
        assert torch.equal(bits(o[side]), bits(out)) and torch.equal(bits(l[1 - side]), bits(lse))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_merge_leaves_out_a_side_without_keys(dtype):
    """lse -inf: whatever out holds; both: 0 and -inf.  The other side's row comes through as it is."""
    inf, nan = float("inf"), float("nan")
    oa = torch.full((4, 64), 1.5, dtype=DTYPES[dtype], device="cuda")
    ob = torch.full((4, 64), -2.5, dtype=DTYPES[dtype], device="cuda")
    la, lb = torch.tensor([3.0, -inf, -inf, nan], device="cuda"), torch.tensor([-inf, 700.0, -inf, 0.0], device="cuda")
    oa[1:3], ob[0], ob[2] = nan, inf, inf
    out, lse = pdec.merge_states(oa, la, ob, lb)
    assert (out[0] == 1.5).all() and (out[1] == -2.5).all() and (out[2] == 0).all() and torch.isnan(out[3]).all()
    assert lse[:3].tolist() == [3.0, 700.0, -inf] and torch.isnan(lse[3])


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_a_video_served_from_pages(cache):
    """A long prefix prefilled in chunks (append, then attend), read back for the dense entry points, and the
    event-parallel step on the pages: attention over the shared prefix and over the streams' own rows, joined.
    Checked against the dense step on the rows read back, and against 64 bits."""
    H_q, H_kv, D, page, E, cap = 28, 4, 128, 64, 6, 40
    chunks = [129, 1, 500, 64, 77]
    L = sum(chunks)
    g = torch.Generator().manual_seed(9)
    k_all, v_all = (torch.randn((L, H_kv, D), generator=g).mul(s).bfloat16() for s in (1.0, 0.5))
    q_all = torch.randn((L, H_q, D), generator=g).mul(1.5).bfloat16()
    c = Paged([L], [L], H_q, H_kv, D, page, "bf16", cache, seed=30)
    P = c.vals["k"].shape[0]
    typ = torch.float8_e4m3fn if cache == "e4m3" else torch.bfloat16
    kp, vp = (torch.zeros((P, page, H_kv, D), dtype=torch.bfloat16, device="cuda").to(typ) for _ in "kv")
    sc = dict(zip(("k_scales", "v_scales"), (torch.zeros((P, H_kv, page), dtype=torch.uint8, device="cuda") for _ in "kv"))) \
        if cache == "e4m3" else {}
    table, lens = i32(c.table), [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2)]
    if cache == "e4m3":
        for name, x in (("k", k_all), ("v", v_all)):
            b, byte = quantise(x.float().numpy())
            c.vals[name][:] = 0
            for t in range(L):
                c.vals[name][c.table[0, t // page], t % page] = e4m3_values(b[t]) * 2.0 ** (byte[t].astype(float) - 127)[:, None]
    else:
        for name, x in (("k", k_all), ("v", v_all)):
            for t in range(L):
                c.vals[name][c.table[0, t // page], t % page] = x[t].double().numpy()
    c.q = q_all.float().numpy()
    ref = c.reference()
    at, outs, lses = 0, [], []
    for n in chunks:
        cu = i32([0, n])
        pdec.paged_kv_append(k_all[at:at + n].cuda(), v_all[at:at + n].cuda(), kp, vp, table, cu, lens[0], lens[1], **sc)
        o, l = pdec.paged_attn(q_all[at:at + n].cuda(), kp, vp, table, cu, lens[1], **sc)
        outs.append(o)
        lses.append(l)
        lens.reverse()
        at += n
    compare("bf16", torch.cat(outs), torch.cat(lses), ref, "chunked prefill")

    kd, vd = pdec.paged_kv_read(kp, vp, table, lens[0], i32([0, L]), num_rows=L, **sc)
    ke, ve = (torch.randn((E, cap, H_kv, D), generator=g).mul(s).bfloat16().cuda() for s in (1.0, 0.5))
    ev = i32([3, 40, 0, 1, 17, 40])
    q = torch.randn((E, H_q, D), generator=g).mul(1.5).bfloat16().cuda()
    dense_o, dense_l = pdec.attn_step(q, kd, vd, ke, ve, ev, i32([L]))
    po, pl = pdec.paged_attn(q, kp, vp, table, i32([0, E]), lens[0], causal=False, **sc)
    oo, ol = pdec.attn_step(q, kd[:0], vd[:0], ke, ve, ev, i32([0]))
    o, l = pdec.merge_states(po, pl, oo, ol)
    live = (ev > 0).cpu().numpy()
    # the definition: all the prefix's keys and the stream's own
    q64, kd64, vd64 = q.double().cpu().numpy(), kd.double().cpu().numpy(), vd.double().cpu().numpy()
    ke64, ve64, ev_h = ke.double().cpu().numpy(), ve.double().cpu().numpy(), ev.tolist()
    for e in range(E):
        if not ev_h[e]:  # an ended stream sees the prefix only in the joined result: its caller leaves it out
            continue
        for h in range(H_q):
            kk = np.concatenate([kd64[:, h // 7], ke64[e, :ev_h[e], h // 7]])
            vv = np.concatenate([vd64[:, h // 7], ve64[e, :ev_h[e], h // 7]])
            z = kk @ q64[e, h] / np.sqrt(D)
            m = z.max()
            p = np.exp(z - m)
            lse = m + np.log(p.sum())
            p /= p.sum()
            spread = (np.abs(kk) @ np.abs(q64[e, h])).max() / np.sqrt(D)
            want, size = p @ vv, p @ np.abs(vv)
            tol_o, tol_l = bounds("bf16", D, want, np.array(lse), size, np.array(spread))
            # each side's out is rounded to bf16 before the join: half a step of at most the larger side's |out|
            side = 2.0 ** -8 * np.maximum(np.abs(po[e, h].double().cpu().numpy()), np.abs(oo[e, h].double().cpu().numpy()))
            assert (np.abs(o[e, h].double().cpu().numpy() - want) <= tol_o + side * 1.01 + 1e-6).all(), (e, h)
            assert abs(float(l[e, h]) - lse) <= tol_l + 2.0 ** -20, (e, h)
            assert (np.abs(dense_o[e, h].double().cpu().numpy() - want) <= 2e-2).all()
    assert (dense_l[torch.from_numpy(live)].cpu() - l[torch.from_numpy(live)].cpu()).abs().max() <= 2e-2


def test_cache_calls_in_a_captured_graph():
    """Append, attend, read and merge captured together, replayed with eager work between."""
    c = Paged([1, 7], [300, 60], 14, 2, 128, 16, "bf16", "e4m3", seed=31).put()
    before = i32([299, 53])
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    k_new, v_new = new_rows(c.T, 2, 128, "bf16", 5).cuda(), new_rows(c.T, 2, 128, "bf16", 6).cuda()

    def step():
        pdec.paged_kv_append(k_new, v_new, c.dev["k_pages"], c.dev["v_pages"], c.dev["block_table"],
                             c.dev["cu_tokens"], before, lens, **c.dev_scales)
        o, l = pdec.paged_attn(c.dev["q"], c.dev["k_pages"], c.dev["v_pages"], c.dev["block_table"],
                               c.dev["cu_tokens"], lens, **c.dev_scales)
        kd, vd = pdec.paged_kv_read(c.dev["k_pages"], c.dev["v_pages"], c.dev["block_table"], lens, i32_cu, num_rows=360,
                                    **c.dev_scales)
        return (o, l, kd, vd, *pdec.merge_states(o, l, o, l))

    i32_cu = i32([0, 300, 360])
    want = [x.clone() for x in step()]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for i in range(4):
        for x in got:
            x.fill_(3.0)
        c.dev["k_pages"].view(torch.uint8)[int(c.table[0, 299 // 16]), 299 % 16] = 0x7F
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, got):
            assert torch.equal(bits(x), bits(y)), i
        step()
