"""Attention over 4-bit paged caches at the ends of the number range, against the definition in 64 bits: NaN values,
large and least ones, under probabilities below float32's range and others."""
import numpy as np
import pytest
import torch

from paged4_util import Paged4, quantise4
from paged_util import HALF_STEP, compare
from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu

TYPES = ["f32", "bf16"]


def far_keys(c, where, nats=136.0):
    """The keys (s, t) get a score `nats` below the others': of 4 in their first element times -nats sqrt(D) / 4."""
    c.q[:, :, 0] = 4
    k = np.random.default_rng(4).standard_normal(c.vals["k"].shape)
    for s, t in where:
        k[c.table[s, t // c.page], t % c.page, :, 0] = -nats * c.D ** 0.5 / 4
    c.set("k", *quantise4(k))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 6, 13, 40])
@pytest.mark.parametrize("D,page", [(128, 32), (64, 64), (64, 16)])
def test_a_nan_value_reaches_the_rows_that_see_it_whatever_its_probability(dtype, n, D, page):
    """NaN blocks of values whose probability, some e^-136, is below float32's range: every row that sees the key has
    NaN in the block's 32 elements and nowhere else, however many tokens share the call.  The last ones belong to
    the last tokens' own keys, which earlier tokens do not see."""
    lens = [700, 333]
    where = [(0, 5), (0, 300), (1, 200), (0, 700 - 1), (1, 333 - n)]
    c = Paged4([n, n], lens, 8, 2, D, page, dtype, seed=33)
    far_keys(c, where)
    c.put()
    o1, l1 = (x.clone() for x in c.attn())
    compare(dtype, o1, l1, c.reference(), "without")
    c.spoil("v", 0, 699, block=1)                 # the last token's: of sequence 0's rows only the last one's
    c.spoil("v", 1, 333 - n, head=1, block=0)     # the first new token's: all rows of sequence 1, head 1
    o2, l2 = c.attn()
    compare(dtype, o2, l2, c.reference(), "own keys")
    nan = np.isnan(o2.float().cpu().numpy())
    want = np.zeros_like(nan)
    want[n - 1, :, 32:64] = True
    want[n:, 4:, :32] = True
    assert np.array_equal(nan, want) and torch.equal(l1, l2)
    for s, t in where[:3]:
        c.spoil("v", s, t, head=t % 2, block=1)
    o3, l3 = c.attn()
    compare(dtype, o3, l3, c.reference(), "all")
    for s, heads in ((0, slice(4, 8)), (0, slice(0, 4)), (1, slice(0, 4))):
        want[s * n:s * n + n, heads, 32:64] = True
    assert np.array_equal(np.isnan(o3.float().cpu().numpy()), want) and torch.equal(l1, l3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 3, 6, 40])
@pytest.mark.parametrize("D,page", [(128, 32), (64, 64)])
@pytest.mark.parametrize("small,large", [(-60, 60), (-60, 0), (0, 60), (None, 60)])
def test_a_probability_of_0_adds_nothing(dtype, n, D, page, small, large):
    """Values of 2^small (None: 0), and of 2^large in keys whose probability, some e^-136, is below float32's range:
    their part of a result, 2^large e^-136, is 2^-136 and less."""
    c = Paged4([n, n], [700, 333], 8, 2, D, page, dtype, seed=33)
    where = [(0, 5), (0, 100), (0, 101), (0, 640), (1, 0), (1, 200)]
    far_keys(c, where)
    v = np.random.default_rng(5).standard_normal(c.vals["v"].shape)
    far = [(c.table[s, t // page], t % page) for s, t in where]
    big = [v[at] * 2.0 ** large for at in far]
    v *= 0.0 if small is None else 2.0 ** small
    for at, x in zip(far, big):
        v[at] = x
    c.set("v", *quantise4(v))
    out, lse = c.attn()
    compare(dtype, out, lse, c.reference(), f"{dtype} {small} {large}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 6, 40])
@pytest.mark.parametrize("D,page", [(128, 32), (64, 64)])
@pytest.mark.parametrize("alike", [True, False])
def test_the_least_scale_is_2_to_minus_127(dtype, n, D, page, alike):
    """A byte of 0, which the append does not write: 6 times 2^-127 in every value's first element of 32, 4 in the next.
    A weighted mean of equal numbers is that number: every p is rounded by half a step at most, and so is the mean, of
    which 2^-7 is left for the sums and for products of small p below 2^-126."""
    c = Paged4([n, n], [300, 133], 8, 2, D, page, dtype, seed=35)
    if alike:
        c.q[:] = 0
    code, byte = np.zeros(c.vals["v"].shape, np.uint8), np.zeros((*c.vals["v"].shape[:3], D // 32), np.uint8)
    code[..., 0::32], code[..., 1::32] = 7, 6
    byte[..., 1::2] = 127  # the other blocks are of 6 and 4
    c.set("v", code, byte)
    out, lse = c.attn()
    o = out.double().cpu().numpy()
    for e, v in ((0, 6.0), (1, 4.0)):
        for i in range(D // 32):
            want = v * (2.0 ** -127 if i % 2 == 0 else 1.0)
            assert (np.abs(o[..., 32 * i + e] - want) <= (2 * HALF_STEP[dtype] + 2.0 ** -7) * want).all()
    assert not o.reshape(*o.shape[:2], -1, 32)[..., 2:].any()
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,H_q,H_kv", [(128, 8, 8), (128, 24, 8), (64, 16, 8)])
@pytest.mark.parametrize("byte", [245, 250, 254])
def test_zeros_under_the_largest_scales_are_zeros(dtype, D, H_q, H_kv, byte):
    """Values of 0 whose scale is 2^118 and more, beside blocks of ordinary ones, under scores that rise by some 2^6
    over a sequence's blocks, as do probabilities relative to those of the keys before.  40 sequences read one's pages."""
    S, L = 40, 2500
    c = Paged4([1], [L], H_q, H_kv, D, 64, dtype, seed=36)
    c.q[:, :, 0] = 4
    k = 0.1 * np.random.default_rng(6).standard_normal(c.vals["k"].shape)
    t = np.arange(L)
    k[c.table[0, t // 64], t % 64, :, 0] = (4.2 * t / L * D ** 0.5 / 4)[:, None]  # 4.2 nats are 2^6
    c.set("k", *quantise4(k))
    v = np.random.default_rng(7).standard_normal(c.vals["v"].shape)
    v[..., 32:64] = 0
    code, b = quantise4(v)
    b[..., 1] = byte
    c.set("v", code, b)
    c.put()
    out, lse = pdec.paged_attn(c.dev["q"].expand(S, -1, -1).contiguous(), c.dev["k_pages"], c.dev["v_pages"],
                               c.dev["block_table"].expand(S, -1).contiguous(), c.i32(np.arange(S + 1)), c.i32([L] * S),
                               max_chunk=1, max_len=L, **c.dev_scales)
    assert not out[..., 32:64].any()
    ref = c.reference()
    for s in (0, 1, 20, S - 1):
        compare(dtype, out[s:s + 1], lse[s:s + 1], ref, f"{dtype} {byte} {s}")
    assert torch.isfinite(out.float()).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 6, 40])
@pytest.mark.parametrize("D,page", [(128, 32), (64, 64)])
@pytest.mark.parametrize("size", [-110, -90, -20, 40, 100, 113])
def test_values_near_the_ends_of_the_range(dtype, n, D, page, size):
    """Values of 2^size with zeros among them, a third of the keys' smaller by 2^5.  2^8 times the sum of a row's
    values stays within float32's range: of 2^113 there are some 22 to a sequence."""
    c = Paged4([n, n], [700, 333], 8, 2, D, page, dtype, seed=37)
    v = np.random.default_rng(8).standard_normal(c.vals["v"].shape)
    if size > 110:
        v[:, np.arange(page) % 32 != 1] = 0
    v[..., ::3] = 0
    v *= 2.0 ** (size - 5.0 * (np.arange(v.shape[1]) % 3 == 0))[None, :, None, None]
    c.set("v", *quantise4(v))
    out, lse = c.attn()
    compare(dtype, out, lse, c.reference(), f"{dtype} {size}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 6, 40])
@pytest.mark.parametrize("D,page", [(128, 32), (64, 64), (64, 16)])
@pytest.mark.parametrize("size", [-110, -90, 0, 100])
def test_hidden_codes_and_scales_of_every_size_do_not_matter(dtype, n, D, page, size):
    """Free pages and rows behind a sequence's end hold any codes under any scales, or zeros: the same bits."""
    got = []
    for junk in (False, True):
        c = Paged4([n, n], [700, 333], 8, 2, D, page, dtype, seed=38, junk=True)
        dead = {x: c.scales[x] == 255 for x in "kv"}  # as junk has them
        v = np.random.default_rng(9).standard_normal(c.vals["v"].shape) * 2.0 ** size
        c.set("v", *quantise4(v))
        rng = np.random.default_rng(10)
        for x in "kv":
            d = np.repeat(dead[x], 16, -1)
            c.scales[x][dead[x]] = rng.choice([0, 1, 20, 127, 180, 245, 250, 254, 255], dead[x].sum()) if junk else 127
            c.raw[x][d] = rng.integers(0, 256, d.sum()) if junk else 0
        got.append(c.attn())
    assert torch.isfinite(got[0][0].float()).all() and got[0][0].any()
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 6, 40])
@pytest.mark.parametrize("D,page", [(128, 32), (64, 64)])
def test_small_values_beside_zeros_under_large_scales(dtype, n, D, page):
    """Values of 2^-100 in all blocks of 32 but the second, zeros under scales of 2^118 to 2^127 there: every element to
    its own precision."""
    c = Paged4([n, n], [700, 333], 8, 2, D, page, dtype, seed=39)
    v = np.random.default_rng(11).standard_normal(c.vals["v"].shape) * 2.0 ** -100
    v[..., 32:64] = 0
    code, byte = quantise4(v)
    byte[..., 1] = np.random.default_rng(12).integers(245, 255, byte[..., 1].shape)
    c.set("v", code, byte)
    out, lse = c.attn()
    assert not out[..., 32:64].any()
    compare(dtype, out, lse, c.reference(), dtype)
