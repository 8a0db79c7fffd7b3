"""Paged caches on the host: what the entry points refuse before anything is enqueued, the length check, the plan."""
import ctypes

import numpy as np
import pytest
import torch

from paged_util import e4m3_values, quantise
from paper_2607_02963_amd import pdec

F32, BF16, E4M3 = pdec.PDEC_DTYPE_F32, pdec.PDEC_DTYPE_BF16, pdec.PDEC_DTYPE_E4M3
FAKE = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(16)]


def dims(**kw):
    d = dict(num_seqs=4, num_tokens=100, H_q=28, H_kv=4, D=128, page_size=64, num_pages=1000, max_pages=128,
             dtype_code=BF16, cache_code=BF16)
    d.update(kw)
    return pdec.make_paged_dims(**d)


BAD = [dict(num_seqs=0), dict(num_tokens=0), dict(H_q=27), dict(H_q=0), dict(H_kv=0), dict(D=96), dict(D=0),
       dict(page_size=8), dict(page_size=48), dict(page_size=2048), dict(page_size=0), dict(page_size=-64),
       dict(num_pages=0), dict(max_pages=0), dict(max_pages=1 << 25), dict(max_chunk=-1), dict(max_len=-1),
       dict(max_len=128 * 64 + 1), dict(dtype_code=E4M3), dict(dtype_code=7), dict(cache_code=F32),
       dict(dtype_code=F32), dict(causal=2), dict(causal=-1), dict(scale=float("nan")), dict(scale=float("inf")),
       dict(H_kv=1 << 16, H_q=1 << 16), dict(num_tokens=(1 << 27) + 1), dict(num_seqs=(1 << 27) + 1)]


@pytest.mark.parametrize("kw", BAD, ids=str)
def test_bad_dims_are_refused_by_every_call(kw):
    d, L = dims(**kw), pdec.lib()
    assert pdec.paged_workspace_size(d) == 0
    b = ctypes.byref(d)
    bad = (pdec.PDEC_ERR_INVALID_ARG, pdec.PDEC_ERR_UNSUPPORTED)
    assert L.pdec_paged_attn(b, *FAKE[:11], 1 << 40, None) in bad
    assert L.pdec_paged_kv_append(b, *FAKE[:10], None) in bad
    assert L.pdec_paged_kv_read(b, *FAKE[:9], None) in bad
    assert L.pdec_query_paged_plan(b, ctypes.byref(pdec.PagedPlan())) in bad
    assert L.pdec_check_paged_lengths(b, FAKE[0], FAKE[1], 1) in bad


def _each_pointer(call, names, optional, codes=(pdec.PDEC_ERR_INVALID_ARG,)):
    """A null and a misaligned pointer in every place."""
    for i, name in enumerate(names):
        for p in (None, ctypes.c_void_p(0x100000 * (i + 1) + 1)):
            if p is None and name in optional:
                continue
            args = list(FAKE[:len(names)])
            args[i] = p
            assert call(args) in codes, (name, p)


@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_bad_pointers_are_refused(cache):
    d, L = dims(cache_code=cache), pdec.lib()
    b, ws = ctypes.byref(d), pdec.paged_workspace_size(d)
    none = () if cache == E4M3 else ("k_scales", "v_scales")

    def without(names, args):  # an unquantised cache's scales are not looked at
        return [x if n not in none else None for n, x in zip(names, args)]

    for fn, names, rest in ((L.pdec_paged_attn, ["q", "k", "v", "k_scales", "v_scales", "table", "cu", "lens", "out", "lse", "ws"],
                             (ws, None)),
                            (L.pdec_paged_kv_append, ["k_new", "v_new", "cu", "table", "lens_in", "lens_out", "k", "v",
                                                      "k_scales", "v_scales"], (None,)),
                            (L.pdec_paged_kv_read, ["k", "v", "k_scales", "v_scales", "table", "lens", "cu", "k_out", "v_out"],
                             (None,))):
        names_checked = [n for n in names if n not in none]
        for name in names_checked:
            i = names.index(name)
            for p in (None, ctypes.c_void_p(0x100000 * (i + 1) + 1)):
                if p is None and name == "lse":
                    continue
                args = without(names, FAKE[:len(names)])
                args[i] = p
                assert fn(b, *args, *rest) == pdec.PDEC_ERR_INVALID_ARG, (fn, name, p)
    args = without(["k_new", "v_new", "cu", "table", "lens_in", "lens_out", "k", "v", "k_scales", "v_scales"], FAKE[:10])
    args[5] = args[4]
    assert L.pdec_paged_kv_append(b, *args, None) == pdec.PDEC_ERR_INVALID_ARG  # lens_out is lens_in
    args = without(["q", "k", "v", "k_scales", "v_scales", "table", "cu", "lens", "out", "lse", "ws"], FAKE[:11])
    assert L.pdec_paged_attn(b, *args, ws - 1, None) == pdec.PDEC_ERR_WORKSPACE


def test_merge_refusals():
    L = pdec.lib()
    names = ["out_a", "lse_a", "out_b", "lse_b", "out", "lse"]
    _each_pointer(lambda a: L.pdec_merge_states(10, 128, BF16, *a, None), names, {"lse"})
    for n, D, t in ((0, 128, BF16), (-1, 128, BF16), (10, 96, BF16), (10, 128, E4M3), (10, 128, 9), (1 << 41, 128, BF16),
                    ((1 << 28) + 1, 128, BF16), ((1 << 29) + 1, 64, F32), ((1 << 63) - 1, 128, F32)):
        assert L.pdec_merge_states(n, D, t, *FAKE[:6], None) in (pdec.PDEC_ERR_INVALID_ARG, pdec.PDEC_ERR_UNSUPPORTED)


@pytest.mark.parametrize("kw", [dict(num_seqs=1 << 25, max_len=64, max_chunk=1), dict(num_seqs=1 << 27, max_chunk=1),
                                dict(num_tokens=1 << 27, max_pages=1 << 20), dict(num_seqs=1 << 20, num_tokens=1 << 20)])
def test_more_work_than_a_launch_counts_is_refused(kw):
    d = dims(**kw)
    assert pdec.paged_workspace_size(d) == 0
    assert pdec.lib().pdec_paged_attn(ctypes.byref(d), *FAKE[:11], 1 << 40, None) == pdec.PDEC_ERR_UNSUPPORTED


def test_length_check():
    d = dims(num_seqs=3, num_tokens=20, max_pages=2, max_chunk=8, max_len=100)
    ok = pdec.check_paged_lengths(d, [0, 8, 8, 16], [100, 0, 50])
    assert ok == pdec.PDEC_OK
    for cu, lens in (([1, 8, 8, 16], [9, 9, 9]), ([0, 8, 7, 16], [9, 9, 9]), ([0, 8, 16, 21], [9, 9, 9]),
                     ([0, 9, 9, 16], [9, 9, 9]), ([0, 8, 8, 16], [101, 9, 9]), ([0, 8, 8, 16], [9, -1, 9])):
        assert pdec.check_paged_lengths(d, cu, lens) == pdec.PDEC_ERR_BAD_LENGTHS, (cu, lens)
    assert pdec.check_paged_lengths(d, [0, 9, 9, 16], [9, 9, 9], attn=False) == pdec.PDEC_OK  # no bound for reads
    with pytest.raises(pdec.PdecError):
        pdec.check_paged_lengths(dims(D=32), [0] * 5, [0] * 4)


def test_binding_refuses_host_tensors_and_wrong_shapes():
    q = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    k = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    table, cu, lens = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        pdec.paged_attn(q, k, k, table, cu, lens)  # not device memory
    with pytest.raises(ValueError):
        pdec.paged_attn(q, k, k, table, cu[:1], lens)
    with pytest.raises(ValueError):
        pdec.paged_kv_append(q[:, :2], q[:, :2], k, k, table, cu, lens, lens[:0])
    with pytest.raises(ValueError):
        pdec.paged_kv_read(k, k, table, lens, cu)  # neither outputs nor num_rows
    with pytest.raises(TypeError):
        pdec.paged_attn(q.half(), k, k, table, cu, lens)
    with pytest.raises(ValueError):
        pdec.merge_states(q, torch.zeros(3, 8), q, torch.zeros(3, 7))


def test_workspace_does_not_grow_with_the_batch_or_the_lengths():
    """Partial states belong to work-groups: at most two each."""
    big = pdec.paged_workspace_size(dims(num_seqs=64, num_tokens=64, max_pages=4096, num_pages=1 << 20))
    small = pdec.paged_workspace_size(dims(num_seqs=4, num_tokens=64, max_pages=4096))
    assert 0 < small and big <= small + (1 << 16)
    assert pdec.paged_workspace_size(dims(max_len=64)) <= 1024  # nothing to cut


def test_the_test_quantiser():
    """Every finite e4m3 value is its own rounding; ties go to even."""
    codes = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    v = e4m3_values(codes)
    got, byte = quantise(np.concatenate([v, [448.0]])[None])
    assert byte[0] == 127 and np.array_equal(got[0, :-1], codes)
    got, _ = quantise(np.array([[448.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, -17.0]]))
    assert e4m3_values(got)[0].tolist() == [448.0, 16.0, 20.0, 0.0, 2.0 ** -8, -16.0]
