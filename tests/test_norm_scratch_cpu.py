"""Which scratch buffer the norm calls of the binding hand to the library, on a stand-in for it (no GPU)."""

import types

import pytest

torch = pytest.importorskip("torch")

import paper_2402_15106_amd as dm  # noqa: E402
from paper_2402_15106_amd import _lib  # noqa: E402

C, G = 8, 2


@pytest.fixture
def lib(monkeypatch):
    """A handle whose library records the scratch address and size of each call; `state` has the stream and
    whether it is captured."""
    monkeypatch.setattr(_lib, "_current_stream", lambda index: state.stream)
    monkeypatch.setattr(_lib, "_capturing", lambda: state.capturing)
    state = types.SimpleNamespace(stream=11, capturing=False, used=[])

    class StandIn:
        def dsmp_group_norm_workspace(self, desc, seg, f, b):
            f._obj.value = b._obj.value = 1000 * seg._obj.n
            return 0

        def dsmp_set_stream(self, h, s):
            return 0

        def dsmp_group_norm_forward(self, *a):
            state.used.append(a[-2:])
            return 0

        dsmp_group_norm_backward = dsmp_group_norm_forward

    h = _lib.Dsmp.__new__(_lib.Dsmp)
    h.lib, h.h, h.device, h._index, h._ws, h._norm_sizes = StandIn(), None, torch.device("cpu"), -1, {}, {}
    h.state = state
    return h


def calls(h, n, **kw):
    """The scratch (address, size) of a forward and of a backward call on n rows."""
    x, d = torch.zeros(n, C), dm.norm_desc(C, G, dm.F32, dm.F32)
    h.state.used.clear()
    _, st = h.dsmp_group_norm_forward(d, x, None, None, **kw)
    h.dsmp_group_norm_backward(d, x, st, None, None, x, **kw)
    return list(h.state.used)


def test_calls_outside_a_capture_share_a_buffer_of_their_stream(lib):
    a = calls(lib, 4)
    assert a[0] == a[1] and calls(lib, 2) == a
    lib.state.stream = 12
    assert calls(lib, 4)[0][0] != a[0][0]


def test_captured_calls_use_no_buffer_that_others_use_or_replace(lib):
    shared = calls(lib, 4)[0][0]
    held = dict(lib._ws)
    lib.state.capturing = True
    captured = calls(lib, 4)
    assert all(p != shared and size >= 4000 for p, size in captured)
    assert lib._ws == held                          # and leaves none behind for calls after the capture
    captured = calls(lib, 9)
    assert lib._ws == held
    lib.state.capturing = False
    assert calls(lib, 4)[0][0] == shared


def test_the_callers_own_scratch(lib):
    d = dm.norm_desc(C, G, dm.F32, dm.F32)
    assert lib.dsmp_group_norm_workspace(d, 5) == (5000, 5000)
    ws = torch.empty(5000, dtype=torch.uint8)
    for lib.state.capturing in (False, True):
        assert calls(lib, 5, ws=ws) == [(ws.data_ptr(), 5000)] * 2
    assert not lib._ws
    for bad in (torch.empty(5000), torch.empty(10000, dtype=torch.uint8)[::2], 7):
        with pytest.raises(dm.DsmpError):
            calls(lib, 5, ws=bad)
