"""How the binding takes the segments of the norm calls (no GPU)."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2402_15106_amd as dm  # noqa: E402
from paper_2402_15106_amd import _lib  # noqa: E402


@pytest.fixture(scope="module")
def h():
    h = _lib.Dsmp.__new__(_lib.Dsmp)
    h.h, h.device, h._index = None, torch.device("cpu"), -1
    return h


def test_counts_and_bounds(h):
    for given, want in ((None, 1), (1, 1), (4, 4), (np.int64(6), 6), (12, 12)):
        s = h._segments(12, given)
        assert (s.n, s.n_seg, s.ptr) == (12, want, None)
    ptr = torch.tensor([0, 5, 12], dtype=torch.int32)
    s = h._segments(12, ptr)
    assert (s.n_seg, s.ptr) == (2, ptr.data_ptr())
    assert h._segments(0, 5).n_seg == 5


@pytest.mark.parametrize("given", [2.5, 3.0, "3", [0, 12], -1, 0, 5, 1 << 40, torch.zeros(0, dtype=torch.int32),
                                   torch.zeros(1, dtype=torch.int32), torch.zeros(3), torch.tensor(3, dtype=torch.int32)])
def test_anything_else_is_refused(h, given):
    """Before anything is allocated for it: a fraction is not taken for the whole number below it."""
    with pytest.raises(dm.DsmpError) as e:
        h._segments(12, given)
    assert e.value.status == dm.INVALID_ARG
