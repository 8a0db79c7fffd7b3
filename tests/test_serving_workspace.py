"""The memory that the table calls allocate for themselves is held until the call is enqueued, and none of it twice.  On
the CPU: the library's entry notes what is alive when it is called."""
import weakref

import pytest
import torch

from paper_2607_02963_amd import pdec


@pytest.fixture
def calls(monkeypatch):
    """What a call allocates, and [(entry, arguments, the allocations alive)]."""
    made, seen = [], []

    def empty(stream, shape, dtype, device):
        t = torch.empty(shape, dtype=dtype)
        made.append((weakref.ref(t), t.data_ptr(), t.nbytes))
        return t

    class Library:
        pdec_table_workspace_size = staticmethod(lambda dims: 4096)

        def __getattr__(self, name):
            def entry(*args):
                seen.append((name, args, [(p, n) for ref, p, n in made if ref() is not None]))
                return pdec.PDEC_OK
            return entry

    pdec._table_dims.cache_clear()
    monkeypatch.setattr(pdec, "_empty", empty)
    monkeypatch.setattr(pdec, "_device_of", lambda t, name, rows=True: (-1, None))
    monkeypatch.setattr(pdec, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(pdec, "lib", lambda: Library())
    yield made, seen
    pdec._table_dims.cache_clear()


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("S", [65, 1500])
def test_the_workspace_lives_as_long_as_the_call(calls, S):
    made, seen = calls
    table, free, a, b = i32(S, 4), i32(100), i32(1), i32(1)
    cu = pdec.paged_reserve(i32(S), i32(S), table, free, a, b, page_size=16, num_tokens=500)
    pdec.paged_release(i32(S), table, free, b, a, page_size=16)
    assert [name for name, _, _ in seen] == ["pdec_paged_reserve", "pdec_paged_release"]
    for (name, args, alive), count in zip(seen, (2, 1)):
        ws = (args[-3], args[-2])
        assert ws[1] == 4096 and ws in alive, f"{name}: the workspace is nobody's"
        spans = sorted(alive)
        assert all(p + n <= q for (p, n), (q, _) in zip(spans, spans[1:]))
    assert cu.shape == (S + 1,) and len(made) == 3


def test_a_given_workspace_is_taken(calls):
    made, seen = calls
    ws = torch.empty(5000, dtype=torch.uint8)
    pdec.paged_release(i32(70), i32(70, 4), i32(100), i32(1), i32(1), page_size=16, workspace=ws)
    assert seen[0][1][-3:-1] == (ws.data_ptr(), 5000) and not made
