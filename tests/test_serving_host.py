"""Block tables and rotary positions on the host: what the calls refuse before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_2607_02963_amd import pdec

FAKE = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(20)]
BAD = (pdec.PDEC_ERR_INVALID_ARG, pdec.PDEC_ERR_UNSUPPORTED)
INVALID = pdec.PDEC_ERR_INVALID_ARG


def table_dims(num_seqs=4, num_tokens=100, page_size=64, num_pages=1000, max_pages=128, max_len=0):
    return pdec.TableDims(num_seqs, num_tokens, page_size, num_pages, max_pages, max_len)


@pytest.mark.parametrize("kw", [dict(num_seqs=0), dict(num_seqs=(1 << 20) + 1), dict(num_tokens=0), dict(num_tokens=(1 << 27) + 1),
                                dict(page_size=0), dict(page_size=8), dict(page_size=48), dict(page_size=2048), dict(num_pages=0),
                                dict(max_pages=0), dict(max_pages=1 << 25), dict(max_len=-1), dict(max_len=128 * 64 + 1)], ids=str)
def test_bad_table_dims(kw):
    d, L = ctypes.byref(table_dims(**kw)), pdec.lib()
    assert L.pdec_table_workspace_size(d) == 0
    assert L.pdec_paged_reserve(d, *FAKE[:10], 1 << 40, None) in BAD
    assert L.pdec_paged_release(d, *FAKE[:7], 1 << 40, None) in BAD


def test_bad_table_pointers():
    d, L = ctypes.byref(table_dims(num_seqs=65)), pdec.lib()
    ws = L.pdec_table_workspace_size(d)
    assert ws > 0 and L.pdec_table_workspace_size(ctypes.byref(table_dims(num_seqs=64))) == 0  # none needed
    for fn, names in ((L.pdec_paged_reserve, ["new", "lens", "table", "free", "in", "out", "cu", "positions", "slots", "ws"]),
                      (L.pdec_paged_release, ["keep_from", "keep_len", "table", "free", "in", "out", "ws"])):
        for i, name in enumerate(names):
            off = {"ws": 8, "slots": 4}.get(name, 2)
            for p in (None, ctypes.c_void_p(0x100000 * (i + 1) + off)):
                if p is None and name in ("positions", "slots", "keep_from"):
                    continue
                args = list(FAKE[:len(names)])
                args[i] = p
                assert fn(d, *args, ws, None) == INVALID, (name, p)
        args = list(FAKE[:len(names)])
        assert fn(d, *args, ws - 1, None) == pdec.PDEC_ERR_WORKSPACE
        i = names.index("in")
        args[i + 1] = args[i]  # one array for both counts
        assert fn(d, *args, ws, None) == INVALID
    assert L.pdec_paged_reserve(None, *FAKE[:10], ws, None) == INVALID


def spec(**kw):
    d = dict(head_dim=128, rotary_dim=0, interleaved=0, scaling=0, theta=1e4, factor=2.0, original_len=4096.0, slow_turns=1.0,
             fast_turns=32.0, magnitude=1.0, freqs=None)
    d.update(kw)
    return pdec.RopeSpec(*d.values())


NAN, INF = float("nan"), float("inf")
BAD_SPECS = [dict(head_dim=96), dict(head_dim=0), dict(rotary_dim=-16), dict(rotary_dim=144), dict(rotary_dim=24), dict(rotary_dim=2),
             dict(interleaved=2), dict(interleaved=-1), dict(scaling=-1), dict(scaling=5), dict(theta=0.0), dict(theta=-1.0),
             dict(theta=NAN), dict(theta=INF), dict(scaling=1, factor=0.0), dict(scaling=2, factor=-2.0), dict(scaling=3, factor=NAN),
             dict(scaling=3, original_len=0.0), dict(scaling=3, slow_turns=32.0), dict(scaling=3, fast_turns=INF),
             dict(scaling=3, slow_turns=NAN), dict(magnitude=NAN), dict(magnitude=INF), dict(scaling=4), dict(scaling=4, freqs=0x1004)]


def rope_call(s, T=10, H_q=28, H_k=4, code=pdec.PDEC_DTYPE_BF16, back=0, pos=FAKE[0], q=FAKE[1], qs=28 * 128, qo=FAKE[2],
              qos=28 * 128, k=FAKE[3], ks=4 * 128, ko=FAKE[4], kos=4 * 128):
    return pdec.lib().pdec_rope(s, T, H_q, H_k, code, back, pos, q, qs, qo, qos, k, ks, ko, kos, None)


def append_call(s, dims=None, **kw):
    d = dict(q=FAKE[0], qs=28 * 128, qo=FAKE[1], qos=28 * 128, k=FAKE[2], ks=4 * 128, v=FAKE[3], vs=4 * 128, base=FAKE[4], cu=FAKE[5],
             table=FAKE[6], lens_in=FAKE[7], lens_out=FAKE[8], kp=FAKE[9], vp=FAKE[10], ksc=FAKE[11], vsc=FAKE[12])
    d.update(kw)
    dims = dims or pdec.make_paged_dims(4, 10, 28, 4, 128, 64, 100, 16, pdec.PDEC_DTYPE_BF16, pdec.PDEC_DTYPE_E2M1)
    return pdec.lib().pdec_paged_rope_kv_append(dims, s, *d.values(), None)


@pytest.mark.parametrize("kw", BAD_SPECS, ids=str)
def test_bad_specs(kw):
    assert rope_call(spec(**kw)) in BAD and append_call(spec(**kw)) in BAD


@pytest.mark.parametrize("kw", [dict(T=0), dict(T=-1), dict(T=(1 << 27) + 1), dict(H_q=0), dict(H_q=-1), dict(H_k=-1), dict(code=2),
                                dict(code=3), dict(code=7), dict(back=2), dict(back=-1), dict(qs=28 * 128 - 8), dict(qs=28 * 128 + 4),
                                dict(qs=0), dict(qs=-28 * 128), dict(qos=28 * 128 + 2), dict(ks=504), dict(kos=516),
                                dict(q=FAKE[2], qs=29 * 128), dict(k=FAKE[4], kos=5 * 128), dict(qs=1 << 62)], ids=str)
def test_bad_sizes_and_strides(kw):
    assert rope_call(spec(), **kw) in BAD


def test_bad_rope_pointers():
    for name in ("pos", "q", "qo", "k", "ko"):
        for p in (None, ctypes.c_void_p(0x100002 if name == "pos" else 0x100008)):
            assert rope_call(spec(), **{name: p}) == INVALID, name
    assert rope_call(None) == INVALID
    # float32 rows are whole 16 bytes by fours
    assert rope_call(spec(), code=pdec.PDEC_DTYPE_F32, qs=28 * 128 + 2) == INVALID


def test_bad_arguments_of_the_fused_append():
    off = {"base": 2, "cu": 2, "table": 2, "lens_in": 2, "lens_out": 2}
    for name in ("q", "qo", "k", "v", "base", "cu", "table", "lens_in", "lens_out", "kp", "vp", "ksc", "vsc"):
        for p in (None, ctypes.c_void_p(0x100000 + off.get(name, 8))):
            if p is None and name == "base":
                continue
            assert append_call(spec(), **{name: p}) == INVALID, name
    for kw in (dict(lens_out=FAKE[7]), dict(qs=28 * 128 - 8), dict(ks=4 * 128 + 1), dict(vs=0), dict(qos=5), dict(q=FAKE[1], qs=30 * 128)):
        assert append_call(spec(), **kw) == INVALID, kw
    assert append_call(spec(head_dim=64)) == INVALID  # another width than the cache's
    assert append_call(spec(), pdec.make_paged_dims(4, 10, 27, 4, 128, 64, 100, 16, 1, 1)) == INVALID
    assert append_call(None) == INVALID


def test_the_binding_refuses_what_it_can_see():
    with pytest.raises(ValueError):
        pdec.rope_spec(128, scaling="cubic")
    with pytest.raises(ValueError):
        pdec.rope_spec(128, freqs=torch.zeros(64, dtype=torch.float64))  # not in device memory
    q = torch.zeros((3, 2, 128))
    with pytest.raises(ValueError):  # on the CPU
        pdec.rope(q, None, torch.zeros(3, dtype=torch.int32), pdec.rope_spec(128))
    with pytest.raises(ValueError):
        pdec.paged_reserve(torch.zeros(2, dtype=torch.int32), None, None, None, None, None, page_size=16, num_tokens=1)
