"""4-bit paged caches on the host: what the calls refuse before anything is enqueued, and the plan."""
import ctypes

import numpy as np
import pytest
import torch

from paged4_util import quantise4, values4
from paper_2607_02963_amd import pdec

F32, BF16, E2M1 = pdec.PDEC_DTYPE_F32, pdec.PDEC_DTYPE_BF16, pdec.PDEC_DTYPE_E2M1
FAKE = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(16)]


def dims(**kw):
    d = dict(num_seqs=4, num_tokens=100, H_q=28, H_kv=4, D=128, page_size=64, num_pages=1000, max_pages=128,
             dtype_code=BF16, cache_code=E2M1)
    d.update(kw)
    return pdec.make_paged_dims(**d)


@pytest.mark.parametrize("kw", [dict(dtype_code=E2M1), dict(cache_code=4), dict(D=96), dict(D=32), dict(page_size=8),
                                dict(page_size=2048), dict(max_len=128 * 64 + 1)], ids=str)
def test_bad_dims_are_refused_by_every_call(kw):
    d, L = dims(**kw), pdec.lib()
    assert pdec.paged_workspace_size(d) == 0
    b, bad = ctypes.byref(d), (pdec.PDEC_ERR_INVALID_ARG, pdec.PDEC_ERR_UNSUPPORTED)
    assert L.pdec_paged_attn(b, *FAKE[:11], 1 << 40, None) in bad
    assert L.pdec_paged_kv_append(b, *FAKE[:10], None) in bad
    assert L.pdec_paged_kv_read(b, *FAKE[:9], None) in bad


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_bad_pointers_are_refused(dtype):
    """A null and a misaligned pointer in every place; the scales are 16-byte aligned here."""
    d, L = dims(dtype_code=dtype), pdec.lib()
    b, ws = ctypes.byref(d), pdec.paged_workspace_size(d)
    for fn, names, rest in ((L.pdec_paged_attn, ["q", "k", "v", "k_scales", "v_scales", "table", "cu", "lens", "out", "lse", "ws"],
                             (ws, None)),
                            (L.pdec_paged_kv_append, ["k_new", "v_new", "cu", "table", "lens_in", "lens_out", "k", "v",
                                                      "k_scales", "v_scales"], (None,)),
                            (L.pdec_paged_kv_read, ["k", "v", "k_scales", "v_scales", "table", "lens", "cu", "k_out", "v_out"],
                             (None,))):
        for i, name in enumerate(names):
            off = 4 if name.endswith("scales") else 1
            for p in (None, ctypes.c_void_p(0x100000 * (i + 1) + off)):
                if p is None and name == "lse":
                    continue
                args = list(FAKE[:len(names)])
                args[i] = p
                assert fn(b, *args, *rest) == pdec.PDEC_ERR_INVALID_ARG, (name, p)
    assert L.pdec_paged_attn(b, *FAKE[:11], ws - 1, None) == pdec.PDEC_ERR_WORKSPACE


def test_the_binding_refuses_other_shapes_and_types():
    """On the CPU the first check that a call reaches is the device's; the dims' come before it."""
    q, table = torch.zeros((3, 8, 64), dtype=torch.bfloat16), torch.zeros((2, 5), dtype=torch.int32)
    k = torch.zeros((9, 2, 16, 32), dtype=torch.uint8)
    d = pdec.paged_dims_of(q, k, table)
    assert (d.num_pages, d.page_size, d.num_kv_heads, d.head_dim, d.cache_dtype) == (9, 16, 2, 64, E2M1)
    with pytest.raises(TypeError):
        pdec.paged_dims_of(q, k.to(torch.int8), table)
    with pytest.raises(ValueError):
        pdec.paged_dims_of(q, k[0], table)
    with pytest.raises(ValueError):
        pdec.paged_attn(q, k, k, table, None, None)


@pytest.mark.parametrize("D,n,want", [(128, 1, 16), (128, 4, 32), (64, 1, 16), (64, 3, 32), (64, 6, 48), (128, 6, 48), (64, 9, 64)])
def test_the_rows_of_an_item(D, n, want):
    plan = pdec.query_paged_plan(dims(D=D, num_tokens=4 * n, max_chunk=n))
    assert plan["rows_few"] == want and plan["rows_many"] == 0


def test_the_definition_of_the_tests():
    """The nearest of two neighbours everywhere, the even code at ties, the least power that holds the largest."""
    x = np.zeros((3, 64))
    x[0, :8] = [6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5]
    x[1, :4], x[1, 32:36] = [6.1, -3, 12, .5], [2.0 ** -140, 0, 0, 0]
    x[2, 40] = np.inf
    code, byte = quantise4(x)
    assert byte.tolist() == [[127, 127], [128, 1], [127, 255]]
    v = values4(code, byte)
    assert v[0, :8].tolist() == [6, 0, 1, 1, 2, 2, 4, 4] and v[1, :4].tolist() == [6, -3, 12, 0]
    assert np.isnan(v[2, 32:]).all() and not v[2, :32].any()
