"""Sizes of the paged calls whose products pass 64 bits, on the host: refused, not taken by what is left of the product."""
import ctypes

import pytest

from paper_2607_02963_amd import pdec

F32, BF16, E4M3 = pdec.PDEC_DTYPE_F32, pdec.PDEC_DTYPE_BF16, pdec.PDEC_DTYPE_E4M3


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (F32, E4M3), (BF16, BF16), (BF16, E4M3)])
@pytest.mark.parametrize("H_q,T,max_len", [
    (1 << 29, 1 << 27, 8190 * 64),   # 2^51 + 1 row groups by 2^13 units: 2^64 and a little
    (1 << 29, 1 << 27, 8187 * 64),
    (1 << 30, 1 << 27, 4094 * 64),
    (1 << 29, 1 << 26, 16376 * 64),
])
def test_a_unit_count_past_64_bits_is_refused(dtype, cache, H_q, T, max_len):
    d = pdec.make_paged_dims(1, T, H_q, 1, 64, 64, 1000, 16384, dtype, cache, max_chunk=1, max_len=max_len)
    assert pdec.paged_workspace_size(d) == 0
    plan = pdec.PagedPlan()
    assert pdec.lib().pdec_query_paged_plan(ctypes.byref(d), ctypes.byref(plan)) == pdec.PDEC_ERR_UNSUPPORTED


@pytest.mark.parametrize("S,taken", [(818, True), (819, True), (820, False)])
def test_the_largest_unit_count_that_is_taken(S, taken):
    """(T G / rows + S) H_kv (units + pad + 1) up to 2^30 - 1: here (S / 4 + S) (2^20 + 2), 1023 and 1025 groups."""
    d = pdec.make_paged_dims(S, S, 4, 1, 64, 64, 1 << 20, 1 << 20, F32, F32, max_chunk=1)
    assert (pdec.paged_workspace_size(d) > 0) == taken
