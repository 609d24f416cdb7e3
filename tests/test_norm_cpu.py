"""Host side of the norm and checkpoint calls: workspace sizes and refusals, no GPU."""

import ctypes

import pytest


@pytest.fixture(scope="module")
def dm():
    import paper_2402_15106_amd as dm
    dm.load_library()
    return dm


def _ws(dm, desc, n, n_seg, ptr=None):
    f, b = ctypes.c_size_t(), ctypes.c_size_t()
    seg = dm._lib.CSegments(n, n_seg, ptr)
    st = dm.load_library().dsmp_group_norm_workspace(ctypes.byref(desc), ctypes.byref(seg), ctypes.byref(f),
                                                     ctypes.byref(b))
    return st, f.value, b.value


def test_workspace_covers_the_pieces(dm):
    for n, C, G, k in [(1, 1, 1, 1), (1000, 32, 8, 1), (262144, 128, 32, 1), (99991, 64, 16, 37), (512, 512, 512, 4)]:
        ptr = ctypes.c_void_p(16) if n % k else None          # never read on the host
        st, f, b = _ws(dm, dm.norm_desc(C, G, dm.F32, dm.BF16), n, k, ptr)
        assert st == dm.OK and b >= f
        if not (ptr is None and k == n):
            assert f >= (k + 1) * G * 8                       # at least one chunk, and a piece more for each segment
        assert b >= 2 * C * 4


def test_workspace_refuses(dm):
    ok = dm.norm_desc(32, 4, dm.F32, dm.F32, dm.ACT_GELU)
    assert _ws(dm, ok, 100, 10)[0] == dm.OK
    assert _ws(dm, ok, 100, 3)[0] == dm.INVALID_ARG
    assert _ws(dm, ok, -1, 1)[0] == dm.INVALID_ARG
    assert _ws(dm, ok, 100, 0)[0] == dm.INVALID_ARG
    assert _ws(dm, ok, 1 << 31, 1)[0] == dm.UNSUPPORTED
    assert _ws(dm, dm.norm_desc(513, 1, dm.F32, dm.F32), 10, 1)[0] == dm.UNSUPPORTED
    for bad in (dm.norm_desc(32, 3, dm.F32, dm.F32), dm.norm_desc(0, 1, dm.F32, dm.F32),
                dm.norm_desc(32, 4, 5, dm.F32), dm.norm_desc(32, 4, dm.F32, dm.F32, 4),
                dm.norm_desc(32, 4, dm.F32, dm.F32, 0, float("inf"))):
        assert _ws(dm, bad, 10, 1)[0] == dm.INVALID_ARG
    lib = dm.load_library()
    assert lib.dsmp_group_norm_workspace(None, None, None, None) == dm.INVALID_ARG


def test_null_handle_is_rejected(dm):
    lib = dm.load_library()
    assert lib.dsmp_checkpoint_store(None, None, 0, 1, 0, 1, None) == dm.INVALID_ARG
    assert lib.dsmp_checkpoint_load(None, None, 0, 1, None, 0, 1) == dm.INVALID_ARG
    assert lib.dsmp_group_norm_restore(None, None, None, None, None, None, None, None, 1) == dm.INVALID_ARG
    assert lib.dsmp_group_norm_forward(None, None, None, None, 1, None, 1, None, 1, None, None, None, 1, None, None, None,
                                       0) == dm.INVALID_ARG
    assert lib.dsmp_group_norm_backward(None, None, None, None, 1, None, None, None, None, None, 1, None, 1, None, 1, None,
                                        None, 0, None, 0) == dm.INVALID_ARG
