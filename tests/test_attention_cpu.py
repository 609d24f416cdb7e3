"""Host side of the rotation and attention calls: workspace sizes, refusals, frequencies, no GPU."""

import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2402_15106_amd as dm  # noqa: E402
from paper_2402_15106_amd import _lib  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    return dm.load_library()


def attention_ws(lib, desc, q, k):
    f, b = ctypes.c_size_t(), ctypes.c_size_t()
    st = lib.dsmp_attention_workspace(desc, _lib.CSegments(*q), _lib.CSegments(*k), ctypes.byref(f), ctypes.byref(b))
    return st, f.value, b.value


def test_attention_workspace(lib):
    d = dm.attention_desc(8, 2, 64, dm.BF16)
    st, f, b = attention_ws(lib, dm.attention_desc(8, 8, 64, dm.BF16), (16384, 1, None), (16384, 1, None))
    assert st == dm.OK and f == 0 and b == 2 * 16384 * 8 * 4                 # the tiles fill the card: no parts to join
    st, f, b = attention_ws(lib, d, (5, 1, None), (262144, 1, None))
    assert st == dm.OK and f >= 2 * 5 * 8 * 66 * 4 and b >= 2 * 5 * 8 * 64 * 4    # two parts at least
    st, f, b = attention_ws(lib, d, (5, 1, None), (100, 1, None))
    assert st == dm.OK and f == 0 and 2 * 5 * 8 * 4 <= b <= 512
    assert attention_ws(lib, d, (0, 3, None), (0, 3, None)) == (dm.OK, 0, 0)


@pytest.mark.parametrize("change,status", [
    (dict(heads=0), dm.INVALID_ARG), (dict(heads=3), dm.INVALID_ARG), (dict(heads=512, kv_heads=512), dm.UNSUPPORTED),
    (dict(head_dim=12), dm.UNSUPPORTED), (dict(head_dim=136), dm.UNSUPPORTED), (dict(head_dim=0), dm.INVALID_ARG),
    (dict(dtype=2), dm.INVALID_ARG), (dict(dim=4), dm.INVALID_ARG), (dict(dim=-1), dm.INVALID_ARG),
    (dict(scale=float("nan")), dm.INVALID_ARG), (dict(scale=1e-30), dm.UNSUPPORTED), (dict(scale=-1e30), dm.UNSUPPORTED),
    (dict(cap=1e-30), dm.UNSUPPORTED), (dict(cap=1025.0), dm.UNSUPPORTED), (dict(cap=1024.0), dm.OK), (dict(cap=1e6, dtype=dm.F32), dm.OK),
    (dict(scale=2.0 ** 62, cap=2.0 ** -62), dm.UNSUPPORTED), (dict(scale=2.0 ** 60, cap=2.0 ** -60), dm.OK), (dict(scale=0.0), dm.OK), (dict(scale=-0.1), dm.OK), (dict(cap=-1.0), dm.INVALID_ARG), (dict(cap=float("inf")), dm.INVALID_ARG)])
def test_attention_refuses_descriptors(lib, change, status):
    args = {**dict(heads=4, kv_heads=2, head_dim=64, dtype=dm.BF16, dim=2, scale=0.1, cap=0.0), **change}
    assert attention_ws(lib, dm.attention_desc(**args), (10, 1, None), (10, 1, None))[0] == status


def test_attention_refuses_segments(lib):
    d = dm.attention_desc(4, 2, 64, dm.BF16)
    for q, k, status in (((10, 3, None), (10, 3, None), dm.INVALID_ARG), ((10, 2, None), (10, 1, None), dm.INVALID_ARG),
                         ((-1, 1, None), (1, 1, None), dm.INVALID_ARG), ((4, 0, None), (4, 0, None), dm.INVALID_ARG),
                         ((1 << 31, 1, None), (1, 1, None), dm.UNSUPPORTED), ((1, 1, None), (1 << 31, 1, None), dm.UNSUPPORTED),
                         (((1 << 30) + 8, 1, None), (1, 1, None), dm.UNSUPPORTED)):     # 2^31 rows of heads that share keys
        assert attention_ws(lib, d, q, k)[0] == status, (q, k)
    assert lib.dsmp_attention_workspace(None, None, None, None, None) == dm.INVALID_ARG


def test_rotation_refuses(lib):
    def ws(n, *a, **kw):
        nb = ctypes.c_size_t()
        return lib.dsmp_qk_rotate_workspace(dm.rotate_desc(*a, **kw), n, ctypes.byref(nb)), nb.value

    assert ws(10, 4, 2, 64, dm.F32, 64)[0] == dm.OK and ws(10, 4, 2, 64, dm.F32, 64)[1] >= 2 * 64 * 4
    assert ws(10, 4, 2, 64, dm.F32, 64, norm=False) == (dm.OK, 0)
    assert ws(10, 4, 3, 64, dm.F32, 0)[0] == dm.OK                       # the heads of both need not divide here
    for n, a, kw, status in ((-1, (4, 2, 64, dm.F32, 64), {}, dm.INVALID_ARG), (1 << 31, (4, 2, 64, dm.F32, 64), {}, dm.UNSUPPORTED),
                             (1, (0, 2, 64, dm.F32, 64), {}, dm.INVALID_ARG), (1, (257, 2, 64, dm.F32, 64), {}, dm.UNSUPPORTED),
                             (1, (4, 2, 60, dm.F32, 60), {}, dm.UNSUPPORTED), (1, (4, 2, 64, 5, 64), {}, dm.INVALID_ARG),
                             (1, (4, 2, 64, dm.F32, 66), {}, dm.INVALID_ARG), (1, (4, 2, 64, dm.F32, 64), dict(axes=3), dm.INVALID_ARG),
                             (1, (4, 2, 64, dm.F32, 64), dict(axes=4), dm.INVALID_ARG), (1, (4, 2, 64, dm.F32, 63), {}, dm.INVALID_ARG),
                             (1, (4, 2, 64, dm.F32, 64), dict(layout=7), dm.INVALID_ARG), (1, (4, 2, 64, dm.F32, 64), dict(eps=-1.0), dm.INVALID_ARG),
                             (1, (4, 2, 64, dm.F32, 64), dict(amplitude=float("inf")), dm.INVALID_ARG)):
        assert ws(n, *a, **kw)[0] == status, (n, a, kw)


def test_null_handle_is_rejected(lib):
    z = (None, 0)
    assert lib.dsmp_qk_rotate_forward(None, None, 1, *z, *z, None, None, None, None, *z, *z) == dm.INVALID_ARG
    assert lib.dsmp_qk_rotate_backward(None, None, 1, *z, *z, None, None, None, None, *z, *z, *z, *z, None, None, 0, None,
                                       0) == dm.INVALID_ARG
    assert lib.dsmp_attention_forward(None, None, None, None, *z, *z, *z, None, None, None, *z, None, None, 0) == dm.INVALID_ARG
    assert lib.dsmp_attention_backward(None, None, None, None, *z, *z, *z, None, None, None, *z, None, *z, *z, *z, *z, None,
                                       0) == dm.INVALID_ARG


def test_frequencies():
    f = dm.rotary_frequencies(8, base=16.0)
    assert torch.equal(f, torch.tensor([1.0, 0.5, 0.25, 0.125]))
    assert torch.equal(dm.rotary_frequencies(24, axes=3, base=16.0), f.repeat(3))
    assert torch.equal(dm.rotary_frequencies(8, base=16.0, factor=4.0), f / 4)
    # over a range of 40 pi: 20, 10, 5 and 2.5 turns; kept from 15 on, a quarter up to 5, half way at 10
    g = dm.rotary_frequencies(8, base=16.0, factor=4.0, extent=40 * math.pi, slow=5.0, fast=15.0)
    assert torch.allclose(g, torch.tensor([1.0, 0.5 * (0.5 + 0.125), 0.0625, 0.03125]), rtol=1e-6)
    assert dm.rotary_frequencies(0).numel() == 0
    for bad in (dict(rot=6, axes=2), dict(rot=8, axes=0), dict(rot=-2), dict(rot=8, base=0.0), dict(rot=8, factor=0.0),
                dict(rot=8, extent=-1.0), dict(rot=8, extent=1.0, slow=3.0, fast=2.0)):
        with pytest.raises(dm.DsmpError) as e:
            dm.rotary_frequencies(**bad)
        assert e.value.status == dm.INVALID_ARG


class StandIn:
    """Records the scratch of each call; every size is a thousand bytes a row."""

    def __init__(self):
        self.used = []

    def dsmp_set_stream(self, h, s):
        return 0

    def dsmp_attention_workspace(self, desc, qs, ks, f, b):
        f._obj.value = b._obj.value = 1000 * qs.n
        return 0

    def dsmp_qk_rotate_workspace(self, desc, n, b):
        b._obj.value = 1000 * n
        return 0

    def call(self, *a):
        self.used.append(a[-2:])
        return 0

    dsmp_attention_forward = dsmp_attention_backward = dsmp_qk_rotate_backward = call


def test_scratch_of_captured_calls_is_their_own(monkeypatch):
    state = dict(capturing=False)
    monkeypatch.setattr(_lib, "_current_stream", lambda index: 11)
    monkeypatch.setattr(_lib, "_capturing", lambda: state["capturing"])
    h = _lib.Dsmp.__new__(_lib.Dsmp)
    h.lib, h.h, h.device, h._index, h._ws, h._attn_sizes = StandIn(), None, torch.device("cpu"), -1, {}, {}
    d, r = dm.attention_desc(1, 1, 8, dm.F32), dm.rotate_desc(1, 1, 8, dm.F32, 0)

    def calls(n, **kw):
        x, g = torch.zeros(n, 8), torch.ones(8)
        h.lib.used.clear()
        out, lse = h.dsmp_attention_forward(d, x, x, x, **kw)
        h.dsmp_attention_backward(d, x, x, x, out, lse, x, **kw)
        h.dsmp_qk_rotate_backward(r, x, x, g, g, None, None, x, x, **kw)
        return list(h.lib.used)

    shared = calls(4)
    assert shared[0] == shared[1] != shared[2] and calls(2) == shared
    held = dict(h._ws)
    state["capturing"] = True
    assert all(p not in (shared[0][0], shared[2][0]) and size >= 9000 for p, size in calls(9)) and h._ws == held
    ws = torch.empty(9000, dtype=torch.uint8)
    assert calls(9, ws=ws) == [(ws.data_ptr(), 9000)] * 3


def test_scratch_of_calls_that_differ_in_type_or_scores_alone():
    """The way a call is cut depends on how long its products and scores take, so its scratch does too."""
    h = _lib.Dsmp.__new__(_lib.Dsmp)
    h.lib, h.h, h._index, h._attn_sizes = dm.load_library(), None, -1, {}
    differ = 0
    for n, nk in ((5, 262144), (600, 9000), (4096, 4096), (3000, 40000)):
        seen = set()
        for dtype in (dm.F32, dm.BF16):
            for dim, cap in ((0, 0.0), (3, 0.0), (2, 9.0)):
                d = dm.attention_desc(8, 2, 64, dtype, dim=dim, cap=cap)
                st, f, b = attention_ws(h.lib, d, (n, 1, None), (nk, 1, None))
                assert st == dm.OK and h.dsmp_attention_workspace(d, n, nk) == (f, b), (n, nk, dtype, dim, cap)
                seen.add((f, b))
        differ += len(seen) > 1
    assert differ        # else this test shows nothing
