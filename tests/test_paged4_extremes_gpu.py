"""Attention over 4-bit paged caches at the ends of the number range, against the definition in 64 bits: NaN values,
and large ones, under probabilities below float32's range."""
import numpy as np
import pytest
import torch

from paged4_util import Paged4, quantise4
from paged_util import compare

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
