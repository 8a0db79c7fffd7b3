"""Writing to 4-bit paged caches and reading them back."""
import numpy as np
import pytest
import torch

from paged4_util import MAGNITUDES, Paged4, pack, quantise4, unpack, values4
from paged_util import DTYPES
from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


def pool(P, H_kv, page, D):
    return [torch.zeros((P, H_kv, page, w), dtype=torch.uint8, device="cuda") for w in (D // 2, D // 2, D // 32, D // 32)]


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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,before,H_kv,D,page", CASES)
def test_append_writes_the_rows_and_nothing_else(dtype, n, before, H_kv, D, page):
    lens = [a + b for a, b in zip(n, before)]
    c = Paged4(n, lens, H_kv, H_kv, D, page, dtype, seed=20, pad=3, junk=True).put()
    g = torch.Generator().manual_seed(1)
    new = {x: torch.randn((c.T, H_kv, D), generator=g).mul(0.7).to(DTYPES[dtype]) for x in "kv"}
    out_lens = torch.full((len(n),), -7, dtype=torch.int32, device="cuda")
    lens_in = i32(before)
    for x in "kv":
        code, byte = quantise4(new[x].float().numpy())
        for s in range(len(n)):
            for i in range(n[s]):
                t, row = before[s] + i, int(c.cu[s]) + i
                p, r = c.table[s, t // page], t % page
                c.raw[x][p, :, r], c.scales[x][p, :, r] = pack(code[row]), byte[row]
    pdec.paged_kv_append(new["k"].cuda(), new["v"].cuda(), c.dev["k_pages"], c.dev["v_pages"], c.dev["block_table"],
                         c.dev["cu_tokens"], lens_in, out_lens, **c.dev_scales)
    assert out_lens.tolist() == lens and lens_in.tolist() == before
    for x in "kv":
        assert np.array_equal(c.dev[x + "_pages"].cpu().numpy(), c.raw[x])
        assert np.array_equal(c.dev_scales[x + "_scales"].cpu().numpy(), c.scales[x])


def test_append_leaves_what_does_not_fit_and_drops_rows_without_a_page():
    """Sequence 0 is one row short, 1 has a bad length, 2 misses the page of its third row, 3 fits exactly."""
    k, v, ks, vs = pool(8, 2, 16, 64)
    table = i32([[0, 1], [2, 3], [4, -1], [5, 6]])
    new = torch.ones((14, 2, 64), device="cuda")
    lens_out = torch.zeros(4, dtype=torch.int32, device="cuda")
    pdec.paged_kv_append(new, 2 * new, k, v, table, i32([0, 5, 7, 11, 14]), i32([28, -3, 14, 29]), lens_out,
                         k_scales=ks, v_scales=vs)
    assert lens_out.tolist() == [28, -3, 18, 32]
    want = torch.zeros(8, 16)
    want[4, 14:] = 1
    want[6, 13:] = 1
    # 1 = 4 * 2^-2, code 6; 2 = 4 * 2^-1
    for pages, scales, byte in ((k, ks, 125), (v, vs, 126)):
        for h in range(2):
            assert torch.equal(pages[:, h].cpu(), (0x66 * want).to(torch.uint8)[..., None].expand(8, 16, 32))
            assert torch.equal(scales[:, h].cpu(), (byte * want).to(torch.uint8)[..., None].expand(8, 16, 2))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_quantisation_of_hard_rows(dtype, D):
    """Ties, every binade of a block, subnormal and largest values, zeros, infinities and NaN, exact powers."""
    tiny = 2.0 ** -149 if dtype == "f32" else 2.0 ** -133
    rows = [np.zeros(D), np.full(D, 6.0), np.full(D, 6.0) * 2.0 ** 125, np.full(D, 6.015625), np.full(D, 1.5), np.full(D, tiny),
            np.linspace(-1, 1, D) * 2.0 ** -126, np.full(D, -3.3e38), 6.0 * 2.0 ** -np.arange(D), -np.zeros(D),
            np.where(np.arange(D) % 40 == 0, np.inf, 1.5), np.where(np.arange(D) == 33, np.nan, -np.arange(D) * 1.0),
            np.full(D, -np.inf), np.full(D, np.nan), np.where(np.arange(D) % 32 == 31, 5.0, tiny),
            2.0 ** np.linspace(-130, 127, D), np.linspace(-8, 8, D) * 2.0 ** 124]
    for e in (-120, -3, 0, 1, 90):
        mids = (MAGNITUDES[:-1] + MAGNITUDES[1:]) / 2
        r = np.resize(np.concatenate([mids, -mids, [6.0, -5.0, 4.5, 3.25]]), D) * 2.0 ** e
        rows += [r, np.nextafter(r.astype(np.float32), np.float32(0)), np.nextafter(r.astype(np.float32), np.float32(np.inf))]
    rng = np.random.default_rng(0)
    rows += list(rng.standard_normal((300, D)) * 2.0 ** rng.uniform(-130, 120, (300, 1)))
    x = torch.tensor(np.array(rows), dtype=torch.float32).to(DTYPES[dtype])
    T = len(rows)
    code, byte = quantise4(x.float().numpy())
    P = (T + 15) // 16
    k, v, ks, vs = pool(P, 1, 16, D)
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    new = x.view(T, 1, D).cuda()
    pdec.paged_kv_append(new, new.neg(), k, v, i32(np.arange(P)[None]), i32([0, T]), i32([0]), lens, k_scales=ks, v_scales=vs)
    assert np.array_equal(ks.view(-1, D // 32)[:T].cpu().numpy(), byte) and torch.equal(ks, vs)
    got, gv = (unpack(p.view(-1, D // 2)[:T].cpu().numpy()) for p in (k, v))
    assert np.array_equal(got & 7, code & 7) and np.array_equal(gv & 7, code & 7)
    some = (code & 7) != 0
    assert np.array_equal(got[some], code[some]) and np.array_equal(gv[some], code[some] ^ 8)
    # a rounding is off by half a step at most: 2^-2 of the value, or 2^-2 of the scale; but magnitudes beyond
    # 6 * 2^125, which become that
    xx, val = x.double().numpy(), values4(got, byte)
    fin = np.repeat(byte != 255, 32, -1) & (np.abs(xx) <= 6 * 2.0 ** 125)
    step = np.repeat(2.0 ** (byte.astype(float) - 129), 32, -1)
    with np.errstate(invalid="ignore"):
        assert (np.abs(val - xx) <= np.maximum(2.0 ** -2 * np.abs(xx), step))[fin].all()
    bad = ~np.isfinite(x.float().numpy()).reshape(T, -1, 32).all(-1)
    assert np.array_equal(byte == 255, bad) and not (got.reshape(T, -1, 32)[bad]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_reading_back_every_code_and_scale(dtype):
    """All 16 codes under every scale byte."""
    D, page, H_kv = 64, 32, 2
    byte = np.arange(256, dtype=np.uint8).reshape(64, 2, 2)  # token, head, block
    code = np.resize(np.concatenate([np.arange(16), np.arange(16)[::-1], np.arange(0, 32, 2) % 16]), (64, 2, D)).astype(np.uint8)
    raw, sc = pack(code), byte
    k = torch.from_numpy(np.ascontiguousarray(raw.reshape(2, page, H_kv, -1).transpose(0, 2, 1, 3))).cuda()
    s = torch.from_numpy(np.ascontiguousarray(sc.reshape(2, page, H_kv, -1).transpose(0, 2, 1, 3))).cuda()
    ko, vo = pdec.paged_kv_read(k, k, i32([[0, 1]]), i32([64]), i32([0, 64]), num_rows=64, dtype=DTYPES[dtype], k_scales=s,
                                v_scales=s)
    v = values4(code, byte)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(v.astype(np.float32)).to(DTYPES[dtype])
    for got in (ko.cpu(), vo.cpu()):
        nan = torch.isnan(want)
        assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,rows,H_kv,D,page", [
    ([1], [1], 1, 64, 16),
    ([100, 0, 33], [100, 0, 33], 4, 128, 16),
    ([100, 7, 64], [40, 20, 64], 2, 128, 64),     # fewer rows than keys, more rows than keys
    ([1000], [1000], 24, 64, 256),
    ([1, 2, 3, 4, 5, 6, 7], [1, 2, 3, 4, 5, 6, 7], 8, 128, 32),
])
def test_read_gives_the_rows_and_zeros(dtype, lens, rows, H_kv, D, page):
    absent = {(0, 1)} if lens[0] > 2 * page else ()
    c = Paged4([0] * len(lens), lens, H_kv, H_kv, D, page, dtype, seed=21, absent=absent, pad=1, junk=True).put()
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


def test_append_and_read_far_into_a_pool():
    """Pages behind 4 GiB of a pool."""
    P, H_kv, page, D = 270000, 4, 64, 128
    k, v, ks, vs = pool(P, H_kv, page, D)
    new = torch.randn((100, H_kv, D), generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).cuda()
    table, lens = i32([[P - 1, P - 7]]), torch.zeros(1, dtype=torch.int32, device="cuda")
    pdec.paged_kv_append(new, -new, k, v, table, i32([0, 100]), i32([0]), lens, k_scales=ks, v_scales=vs)
    ko, vo = pdec.paged_kv_read(k, v, table, lens, i32([0, 100]), num_rows=100, k_scales=ks, v_scales=vs)
    want = torch.from_numpy(values4(*quantise4(new.float().cpu().numpy())))
    assert torch.equal(ko.double().cpu(), want) and torch.equal(vo.double().cpu(), -want)
    assert not k[:P - 7].any() and not ks[:P - 7].any()
