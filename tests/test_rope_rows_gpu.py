"""Rotary positions of a ragged batch against the definition in 64 bits: layouts, partial heads, scalings, strides, far
positions, the gradient; fused with the append to every form of a paged cache; and a serving step's run of it all."""
import math

import numpy as np
import pytest
import torch

from paged4_util import Paged4
from paged_util import DTYPES, HALF_STEP, Paged, compare
from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu

SPECS = [
    dict(head_dim=128, theta=1e6),
    dict(head_dim=64),
    dict(head_dim=128, rotary_dim=64, interleaved=True),
    dict(head_dim=128, rotary_dim=48, theta=5e5, scaling="linear", factor=4.0),
    dict(head_dim=64, rotary_dim=16, interleaved=True, scaling="ntk", factor=2.5),
    dict(head_dim=128, scaling="by_parts", factor=8.0, original_len=4096, magnitude=1.2079),
    dict(head_dim=64, rotary_dim=32, scaling="by_parts", factor=8.0, original_len=8192, slow_turns=1.0, fast_turns=4.0),
    dict(head_dim=128, rotary_dim=96, interleaved=True, magnitude=-0.5),
]


def bits(t):
    return t.contiguous().view({4: torch.int32, 2: torch.int16, 1: torch.uint8}[t.element_size()])


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


def frequencies(head_dim, rotary_dim=None, interleaved=False, theta=10000.0, scaling="none", factor=1.0, original_len=0,
                slow_turns=1.0, fast_turns=32.0, magnitude=1.0):
    R = rotary_dim or head_dim
    if scaling == "ntk":
        theta = theta * factor ** (R / (R - 2))
    f = theta ** (-2.0 * np.arange(R // 2) / R)
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":
        u = np.clip((original_len * f / (2 * math.pi) - slow_turns) / (fast_turns - slow_turns), 0, 1)
        f = u * f + (1 - u) * f / factor
    return f


def turned(x, pos, spec, back=False, f=None):
    """(rows in float64, what bounds an element's error before the last rounding)."""
    R, D, m = spec.get("rotary_dim") or spec["head_dim"], spec["head_dim"], spec.get("magnitude", 1.0)
    f = frequencies(**spec) if f is None else f
    angle = np.asarray(pos, np.float64)[:, None, None] * f
    c, s = m * np.cos(angle), m * np.sin(angle) * (-1 if back else 1)
    i = np.arange(R // 2)
    a, b = (2 * i, 2 * i + 1) if spec.get("interleaved") else (i, i + R // 2)
    x = x.astype(np.float64)
    y, size, far = x.copy(), np.zeros_like(x), np.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a], size[..., b] = np.abs(x[..., a] * c) + np.abs(x[..., b] * s), np.abs(x[..., b] * c) + np.abs(x[..., a] * s)
    far[..., a] = far[..., b] = abs(m) * (np.abs(x[..., a]) + np.abs(x[..., b])) * np.abs(angle)
    return y, size, far


def close(dtype, got, want, what=""):
    """A frequency is off by 2^-47 of itself at most (a power of up to 2^20 from its logarithm in float64), so is the
    angle.  bfloat16: cosines and sines rounded to float32, two products and their sum: 4 half steps (2^-24) of the
    terms.  Then one rounding, or where nothing turns none."""
    y, size, far = want
    tol = HALF_STEP[dtype] * np.abs(y) * (1 + 2.0 ** -6) + 2.0 ** -47 * far + size * (2.0 ** -22 if dtype == "bf16" else 2.0 ** -48) + 1e-38
    tol = np.where(size == 0, 0, tol)
    err = np.abs(got.double().cpu().numpy() - y)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: off by {err[bad].max():.3e} at {np.argwhere(bad)[0]}, {bad.sum()} of {bad.size}, allowed {tol[bad].min():.3e}"


def rows(T, H, D, dtype, seed):
    return torch.randn((T, H, D), generator=torch.Generator().manual_seed(seed)).to(DTYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("spec", SPECS, ids=range(len(SPECS)))
@pytest.mark.parametrize("T,H_q,H_k", [(1, 1, 1), (3, 28, 4), (37, 7, 1), (300, 40, 8), (5, 9, 0), (2100, 5, 3)])
def test_against_64_bits(dtype, spec, T, H_q, H_k):
    D = spec["head_dim"]
    q, k = rows(T, H_q, D, dtype, 1), rows(T, H_k, D, dtype, 2)
    pos = np.random.default_rng(T).integers(-5, 200000, T)
    pos[0] = 0
    for back in (False, True):
        qo, ko = pdec.rope(q.cuda(), k.cuda() if H_k else None, i32(pos), pdec.rope_spec(**spec), backward=back)
        close(dtype, qo, turned(q.double().numpy(), pos, spec, back), f"q {back}")
        if H_k:
            close(dtype, ko, turned(k.double().numpy(), pos, spec, back), f"k {back}")
        else:
            assert ko is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_extreme_positions(dtype):
    spec = dict(head_dim=64)
    pos = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 10 ** 9])
    q = rows(len(pos), 3, 64, dtype, 3)
    qo, _ = pdec.rope(q.cuda(), None, i32(pos), pdec.rope_spec(**spec))
    close(dtype, qo, turned(q.double().numpy(), pos, spec))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("spec", [SPECS[0], SPECS[2], SPECS[6]], ids=str)
def test_strided_rows_in_place_and_a_table(dtype, spec):
    """Slices of one projection turn in place and leave the rest; a table of the same frequencies gives the same."""
    D, T, H_q, H_k = spec["head_dim"], 50, 6, 2
    x = rows(T, H_q + 2 * H_k + 1, D, dtype, 4)
    d = x.cuda()
    q, k = d[:, :H_q], d[:, H_q:H_q + H_k]
    pos = np.arange(T) * 731
    s = pdec.rope_spec(**spec)
    qo, ko = pdec.rope(q, k, i32(pos), s)
    assert qo.is_contiguous() and torch.equal(d.cpu(), x)
    close(dtype, qo, turned(x[:, :H_q].double().numpy(), pos, spec))
    a, b = pdec.rope(q, k, i32(pos), s, q_out=q, k_out=k)
    assert a is q and torch.equal(bits(d[:, :H_q]), bits(qo)) and torch.equal(bits(d[:, H_q:H_q + H_k]), bits(ko))
    assert torch.equal(d[:, H_q + H_k:].cpu(), x[:, H_q + H_k:])
    # out of place into strided rows
    big = torch.full((T, H_q + 3, D), 5.0, dtype=x.dtype, device="cuda")
    pdec.rope(x[:, :H_q].cuda(), None, i32(pos), s, q_out=big[:, 2:2 + H_q])
    assert torch.equal(bits(big[:, 2:2 + H_q]), bits(qo)) and (big[:, :2] == 5).all() and (big[:, 2 + H_q:] == 5).all()
    f = frequencies(**spec) * 1.25
    table = pdec.rope_spec(D, rotary_dim=spec.get("rotary_dim"), interleaved=spec.get("interleaved", False),
                           freqs=torch.from_numpy(f).cuda())
    qt, _ = pdec.rope(x[:, :H_q].cuda(), None, i32(pos), table)
    close(dtype, qt, turned(x[:, :H_q].double().numpy(), pos, spec, f=f))


@pytest.mark.parametrize("T,H", [(1, 3), (4, 1), (5, 3)])
def test_outputs_are_contiguous_whatever_the_rows_strides(T, H):
    """Of one token or head strides say nothing; rows whose heads do not lie one after another are refused."""
    spec, pos = pdec.rope_spec(64), i32(range(T))
    x = rows(2 * T, 2 * H, 64, "f32", 8).cuda()
    want, _ = pdec.rope(x[:T, :H].contiguous(), None, pos, spec)
    for q in (x[:T, :H], x[:T].transpose(0, 1)[:H].transpose(0, 1), x.as_strided((T, H, 64), (2 * H * 64, 64, 1))):
        out, _ = pdec.rope(q, None, pos, spec)
        assert out.is_contiguous() and torch.equal(bits(out), bits(want))
        out, _ = pdec.rope(q, None, pos, spec, stream=torch.cuda.current_stream())
        assert out.is_contiguous() and torch.equal(bits(out), bits(want))
    if H > 1:
        for q in (x[::2, ::2][:T, :H], x.permute(1, 0, 2)[:H].contiguous().permute(1, 0, 2)[:T]):
            with pytest.raises(ValueError, match="one after another"):
                pdec.rope(q, None, pos, spec)


def test_an_output_of_keys_without_keys_is_refused():
    q, pos = rows(2, 3, 64, "f32", 1).cuda(), i32([0, 1])
    with pytest.raises(ValueError, match="k_out"):
        pdec.rope(q, None, pos, pdec.rope_spec(64), k_out=q.clone())


@pytest.mark.parametrize("spec", SPECS, ids=range(len(SPECS)))
def test_the_gradient_is_the_formulas_and_that_of_differences(spec):
    """L = sum w y of float32 rows: dL/dx is the transposed turn of w; and as y is linear in x, (L(x + h e) -
    L(x - h e)) / 2h is dL/dx up to the roundings of y, 2^-24 of each term over h."""
    D, T, H = spec["head_dim"], 4, 2
    s, pos = pdec.rope_spec(**spec), i32([3, 70, 5000, 123456])
    x, w = rows(T, H, D, "f32", 5).cuda(), rows(T, H, D, "f32", 6).cuda()
    dx, _ = pdec.rope(w, None, pos, s, backward=True)
    close("f32", dx, turned(w.double().cpu().numpy(), pos.cpu().numpy(), spec, back=True))
    h = 2.0
    for e in list(range(0, D, 7)) + [D - 1]:
        loss = []
        for sign in (h, -h):
            z = x.clone()
            z[:, :, e] += sign
            loss.append((w.double() * pdec.rope(z, None, pos, s)[0].double()).sum(-1))
        diff = (loss[0] - loss[1]) / (2 * h)
        m = abs(spec.get("magnitude", 1.0)) + 1
        tol = 2.0 ** -23 * m * (w.double().abs() * (x.double().abs().amax() + h)).sum(-1) / h + 2.0 ** -30
        assert ((diff - dx[:, :, e].double()).abs() <= tol).all(), e


FORMS = [("f32", "f32"), ("f32", "e4m3"), ("f32", "e2m1"), ("bf16", "bf16"), ("bf16", "e4m3"), ("bf16", "e2m1")]


def cache_of(cache):
    return Paged4 if cache == "e2m1" else Paged


@pytest.mark.parametrize("dtype,cache", FORMS)
@pytest.mark.parametrize("n,before,H_q,H_kv,page,spec,base", [
    ([1], [0], 4, 1, 16, SPECS[1], False),
    ([1, 1, 1], [0, 63, 64], 28, 4, 64, SPECS[0], True),
    ([5, 0, 33, 1], [11, 7, 100, 0], 6, 2, 16, SPECS[2], True),
    ([300], [17], 8, 8, 128, SPECS[4], False),
    ([70, 130], [1, 30], 9, 3, 32, SPECS[3], True),
    ([0, 2], [5, 1023], 24, 24, 1024, SPECS[6], False),
    ([1030, 0, 1, 2, 0, 0, 1015], [7, 3, 63, 127, 0, 9, 0], 28, 4, 64, SPECS[5], True),
    ([1] * 200, [int(x) for x in np.arange(200) * 7 % 61], 14, 2, 16, SPECS[7], True),
])
def test_the_fused_append_is_rope_and_then_the_append(dtype, cache, n, before, H_q, H_kv, page, spec, base):
    """Bit for bit, for strided rows too; pages, scales and rows of others are left as they were."""
    D = spec["head_dim"]
    lens = [a + b for a, b in zip(n, before)]
    c = cache_of(cache)(n, lens, H_q, H_kv, D, page, dtype, cache, seed=20, pad=3).put()
    x = rows(c.T, H_q + 2 * H_kv, D, dtype, 7).cuda()
    q, k, v = x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
    pos_base = i32(np.arange(len(n)) * 997 + 3) if base else None
    pos = np.concatenate([before[s] + np.arange(n[s]) + (s * 997 + 3 if base else 0) for s in range(len(n))] + [np.zeros(3)])
    s = pdec.rope_spec(**spec)
    args = [c.dev["block_table"], c.dev["cu_tokens"], i32(before)]
    want_q, k_turned = pdec.rope(q, k, i32(pos), s)
    pages = [c.dev[y + "_pages"].clone() for y in "kv"]
    scales = {y: z.clone() for y, z in c.dev_scales.items() if z is not None}
    after = torch.full((len(n),), -7, dtype=torch.int32, device="cuda")
    pdec.paged_kv_append(k_turned, v.contiguous(), *pages, *args, after, **scales)
    after2 = torch.full_like(after, -7)
    out = torch.full((c.T, H_q, D), 9.0, dtype=x.dtype, device="cuda")
    got = pdec.paged_rope_kv_append(q, k, v, c.dev["k_pages"], c.dev["v_pages"], *args, after2, s, pos_base=pos_base, q_out=out,
                                    **c.dev_scales)
    assert got is out and after2.tolist() == after.tolist() == lens
    T = sum(n)
    assert torch.equal(bits(out[:T]), bits(want_q[:T])) and (out[T:] == 9).all()
    for y, w in zip("kv", pages):
        assert torch.equal(bits(c.dev[y + "_pages"].view(torch.uint8)), bits(w.view(torch.uint8)))
    for y, w in scales.items():
        assert torch.equal(c.dev_scales[y], w)
    # in place
    tail = x[T:].clone()
    pdec.paged_rope_kv_append(q, k, v, c.dev["k_pages"], c.dev["v_pages"], *args, after2, s, pos_base=pos_base, q_out=q,
                              **c.dev_scales)
    assert torch.equal(bits(x[:T, :H_q]), bits(want_q[:T])) and torch.equal(bits(x[T:]), bits(tail))


def test_the_fused_append_leaves_what_does_not_fit_and_drops_rows_without_a_page():
    """Sequence 0 is one row short, 1 has a bad length, 2 misses the page of its third row, 3 fits exactly; all their
    queries turn."""
    H, D = 2, 64
    k = torch.zeros((8, 16, H, D), device="cuda")
    v = torch.zeros_like(k)
    lens, cu = [28, -3, 14, 29], [0, 5, 7, 11, 14]
    new, after = rows(14, H, D, "f32", 8).cuda(), i32([0] * 4)
    s = pdec.rope_spec(D)
    out = pdec.paged_rope_kv_append(new, new, new, k, v, i32([[0, 1], [2, 3], [4, -1], [5, 6]]), i32(cu), i32(lens), after, s)
    assert after.tolist() == [28, -3, 18, 32]
    pos = [lens[i] + j for i in range(4) for j in range(cu[i + 1] - cu[i])]
    want, _ = pdec.rope(new, None, i32(pos), s)
    assert torch.equal(out, want)
    kk, vv = torch.zeros_like(k), torch.zeros_like(k)
    kk[4, 14:], kk[6, 13:] = want[7:9], want[11:]
    vv[4, 14:], vv[6, 13:] = new[7:9], new[11:]
    assert torch.equal(k, kk) and torch.equal(v, vv)


def test_calls_on_two_streams_and_in_a_captured_graph():
    s, t = pdec.rope_spec(**SPECS[0]), pdec.rope_spec(**SPECS[2])
    q, pos = rows(500, 28, 128, "bf16", 9).cuda(), i32(np.arange(500))
    want = [pdec.rope(q, None, pos, x)[0] for x in (s, t)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in "ab"]
    got = [pdec.rope(q, None, pos, x, stream=y)[0] for _ in range(3) for x, y in zip((s, t), streams)]
    torch.cuda.synchronize()
    for x, y in zip(3 * want, got):
        assert torch.equal(bits(x), bits(y))
    out = [torch.empty_like(q) for _ in "ab"]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pdec.rope(q, None, pos, s, q_out=out[0])
        pdec.rope(q, None, pos, t, q_out=out[1])
    for i in range(4):
        pos.copy_(i32(np.arange(500) * (i + 1)))
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((s, t), out):
            assert torch.equal(bits(pdec.rope(q, None, pos, x)[0]), bits(y)), i


@pytest.mark.parametrize("dtype,cache", [("bf16", "e2m1"), ("f32", "e2m1"), ("bf16", "bf16"), ("bf16", "e4m3")])
def test_a_serving_loop(dtype, cache):
    """Prefill chunks, then steps of one to three tokens of which some are refused, sequences that end and others that
    come: reserve, append with positions, attend, give back.  The attention is checked against the rows that the cache
    holds, and those against the rotation."""
    rng = np.random.default_rng(11)
    S, H_q, H_kv, D, page, P, cols = 6, 14, 2, 128, 16, 160, 40
    spec = dict(head_dim=D, scaling="by_parts", factor=4.0, original_len=256)
    s = pdec.rope_spec(**spec)
    c = cache_of(cache)([1], [1], H_q, H_kv, D, page, dtype, cache)  # an empty pool's form
    make = lambda w: torch.zeros(w, dtype=torch.uint8, device="cuda")
    if cache == "e2m1":
        pages = [make((P, H_kv, page, D // 2)) for _ in "kv"]
        scales = {x: make((P, H_kv, page, D // 32)) for x in ("k_scales", "v_scales")}
    else:
        kind = torch.float8_e4m3fn if cache == "e4m3" else DTYPES[dtype]
        pages = [torch.zeros((P, page, H_kv, D), dtype=torch.float32, device="cuda").to(kind) for _ in "kv"]
        scales = {x: make((P, H_kv, page)) for x in ("k_scales", "v_scales")} if cache == "e4m3" else {}
    table, free = i32(np.full((S, cols), -1)), i32(rng.permutation(P))
    count, mid = i32([P]), i32([0])
    room = 600
    lens = [0] * S
    history = [np.zeros((0, H_kv, D)) for _ in range(S)]
    for step in range(7):
        n = [int(rng.integers(20, 90)) if t == 0 else int(rng.integers(0, 4)) for t in lens]
        d_lens, after = i32(lens), i32([0] * S)
        pos, slots = i32([0] * room), torch.zeros(room, dtype=torch.int64, device="cuda")
        cu = pdec.paged_reserve(i32(n), d_lens, table, free, count, mid, page_size=page, positions=pos, slots=slots)
        T = sum(n)
        assert cu.tolist() == np.concatenate([[0], np.cumsum(n)]).tolist()
        x = rows(room, H_q + 2 * H_kv, D, dtype, step).cuda()
        q = pdec.paged_rope_kv_append(x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:], *pages, table, cu, d_lens, after, s,
                                      **scales)
        want_q, want_k = pdec.rope(x[:, :H_q], x[:, H_q:H_q + H_kv], pos, s)
        assert torch.equal(bits(q[:T]), bits(want_q[:T])) and after.tolist() == [a + b for a, b in zip(n, lens)]
        close(dtype, want_k[:T], turned(x[:T, H_q:H_q + H_kv].double().cpu().numpy(), pos[:T].cpu().numpy(), spec))
        if cache == dtype:
            flat = pages[0].view(-1, H_kv, D)
            assert torch.equal(bits(flat[slots[:T]]), bits(want_k[:T]))
        out, lse = pdec.paged_attn(q, *pages, table, cu, after, max_chunk=max(n), max_len=cols * page, **scales)
        total = [a + b for a, b in zip(n, lens)]
        dense = pdec.paged_kv_read(*pages, table, after, i32(np.concatenate([[0], np.cumsum(total)])), num_rows=sum(total),
                                   dtype=torch.float32 if dtype == "f32" else torch.bfloat16, **scales)
        ref = Paged(n, total, H_q, H_kv, D, page, dtype)
        ref.q[:] = q[:T].float().cpu().numpy()
        for name, y in zip("kv", dense):
            y, at = y.double().cpu().numpy(), 0
            for i, t in enumerate(total):
                for j in range(t):
                    ref.vals[name][ref.table[i, j // page], j % page] = y[at + j]
                if name == "k":  # what was there has not changed
                    assert np.array_equal(y[at:at + lens[i]], history[i][:lens[i]])
                    history[i] = y[at:at + t]
                at += t
        compare(dtype, out, lse, ref.reference(), f"step {step}")
        lens = [0 if t and rng.random() < 0.15 else t + int(rng.integers(0, a + 1) if t else a) for t, a in zip(lens, n)]
        pdec.paged_release(i32(lens), table, free, mid, count, page_size=page)
        held = sum(-(-t // page) for t in lens)
        assert count.item() == P - held and (table >= 0).sum().item() == held


@pytest.mark.parametrize("fused", [False, True])
def test_more_tokens_than_a_grid_has_threads_in_one_direction(fused):
    """Over four million tokens: the first, the last and some between against the definition, all against each other."""
    T, D, period = (1 << 22) + 77, 64, 1 << 12
    spec = dict(head_dim=D)
    s = pdec.rope_spec(**spec)
    x = rows(period, 1, D, "bf16", 12).cuda().repeat(T // period + 1, 1, 1)[:T].contiguous()
    pos = torch.arange(T, device="cuda", dtype=torch.int32) % period
    if not fused:
        y, _ = pdec.rope(x, None, pos, s)
    else:
        page = 1024
        n = T // page + 1
        table = torch.arange(n, device="cuda", dtype=torch.int32)[:, None].contiguous()
        cu = (torch.arange(n + 1, device="cuda") * page).clamp(max=T).to(torch.int32)
        base = torch.arange(n, device="cuda", dtype=torch.int32) * page % period
        pages = [torch.zeros((n, page, 1, D), dtype=x.dtype, device="cuda") for _ in "kv"]
        lens, after = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        y = pdec.paged_rope_kv_append(x, x, x, *pages, table, cu, lens, after, s, pos_base=base)
        assert torch.equal(after, cu[1:] - cu[:-1])
        assert torch.equal(pages[0].view(-1, 1, D)[:T], y) and torch.equal(pages[1].view(-1, 1, D)[:T], x)
    assert torch.equal(y[period:2 * period], y[:period]) and torch.equal(y[-period - 77:-77], y[:period])
    whole = T // period * period
    assert torch.equal(y[:whole].view(-1, period, D), y[:period].view(1, period, D).expand(T // period, -1, -1))
    close("bf16", y[:64], turned(x[:64].double().cpu().numpy(), np.arange(64), spec))
    tail = np.arange(T - 50, T) % period
    close("bf16", y[-50:], turned(x[-50:].double().cpu().numpy(), tail, spec))
