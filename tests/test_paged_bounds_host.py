"""max_chunk, max_len and scale of the paged calls: a call takes the values that they have when it is made."""
import numpy as np
import pytest
import torch

from paper_2607_02963_amd import pdec

POOL, TABLE = (100, 64, 4, 128), (2, 50)


def dims(max_chunk=0, max_len=0, scale=0.0):
    return pdec._paged_dims(32, 28, POOL, TABLE, pdec.PDEC_DTYPE_BF16, pdec.PDEC_DTYPE_BF16, max_chunk, max_len, 1, scale)


@pytest.mark.parametrize("make", [lambda x: torch.tensor(x), lambda x: np.array(x)], ids=["tensor", "array"])
def test_a_bound_that_is_written_to(make):
    chunk, length, scale = make(5), make(1000), make(0.25)
    d = dims(chunk, length, scale)
    assert (d.max_chunk, d.max_len, d.softmax_scale) == (5, 1000, 0.25)
    chunk += 3
    length += 500
    scale *= 2
    d = dims(chunk, length, scale)
    assert (d.max_chunk, d.max_len, d.softmax_scale) == (8, 1500, 0.5)
    assert dims(8, 1500, 0.5) is d  # the same sizes have the same dims, made once


@pytest.mark.parametrize("kw", [dict(max_len=2 ** 32 + 100), dict(max_chunk=2 ** 32), dict(max_len=-2 ** 32 + 1)], ids=str)
def test_a_bound_beyond_32_bits_is_refused(kw):
    """Its low 32 bits would be another bound, below the lengths it was meant for."""
    with pytest.raises(ValueError):
        dims(**kw)
    with pytest.raises(ValueError):
        pdec.make_paged_dims(2, 32, 28, 4, 128, 64, 100, 50, pdec.PDEC_DTYPE_BF16, pdec.PDEC_DTYPE_BF16, **kw)
