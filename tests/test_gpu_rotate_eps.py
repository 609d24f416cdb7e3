"""dgamma and dx of the rotation's backward pass with eps = 0, against the float64 oracle:
lanes without a row or a head add nothing to the sums (0 times the infinite 1 / rms of no values)."""

import numpy as np
import pytest

from oracle import attention as oa
from tests.helpers import announce
from tests.test_gpu_rotate import Case, env, f64  # noqa: F401

pytestmark = pytest.mark.gpu


def without_eps(env, *args, **kw):  # noqa: F811
    c = Case(env, *args, **kw)
    c.eps = c.desc.eps = 0.0
    return c


# rows times heads that fill no workgroup, a head to a chunk; all three heads of a row in one chunk, taken two by two; five
# heads in chunks of three and two (float32); chunks of three or two heads, the last of one (259 heads); lanes without values
# (heads of 24 and 40)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,H,Hk,hd,rot,axes", [(1, 1, 1, 32, 32, 1), (37, 5, 2, 32, 16, 2), (300, 4, 2, 64, 64, 1), (17001, 2, 1, 128, 128, 2),
                                                (6151, 4, 1, 128, 96, 3), (700, 256, 3, 24, 0, 1), (129, 2, 2, 40, 24, 2)])
@pytest.mark.parametrize("layout", [oa.HALF, oa.INTERLEAVED])
def test_idle_lanes_add_nothing(env, n, H, Hk, hd, rot, axes, layout, dtype):  # noqa: F811
    announce(dtype, n, H, Hk, hd, rot, axes, layout)
    without_eps(env, n, H, Hk, hd, dtype, rot, axes, layout).check()


def test_one_of_both(env):  # noqa: F811
    dm, lib, torch = env
    c = without_eps(env, 301, 4, 3, 64, "bf16", 32, 1, oa.HALF)
    for s, at in (("q", 0), ("k", 1)):
        announce(s)
        x, dy, gamma = ([d[s] if t == s else None for t in "qk"] for d in (c.x, c.dy, c.gamma))
        got = lib.dsmp_qk_rotate_backward(c.desc, *x, *gamma, c.pos, c.freq, *dy)
        assert list(got[2]) == ["dgamma_" + s]
        c.check_backward(got[at], got[2]["dgamma_" + s], s)


def test_a_head_of_zeros_is_lost_alone(env):  # noqa: F811
    """1 / rms of zeros is infinite without eps: that head has no result, the others keep theirs."""
    dm, lib, torch = env
    c = without_eps(env, 50, 3, 1, 32, "f32", 16, 1, oa.HALF)
    q = lib.dsmp_qk_rotate_forward(c.desc, c.x["q"], None, c.gamma["q"], None, c.pos, c.freq)[0]
    gq = lib.dsmp_qk_rotate_backward(c.desc, c.x["q"], None, c.gamma["q"], None, c.pos, c.freq, c.dy["q"], None)[0]
    c.x["q"][7, 32:64] = 0.0
    q2 = lib.dsmp_qk_rotate_forward(c.desc, c.x["q"], None, c.gamma["q"], None, c.pos, c.freq)[0]
    g2 = lib.dsmp_qk_rotate_backward(c.desc, c.x["q"], None, c.gamma["q"], None, c.pos, c.freq, c.dy["q"], None)[0]
    for was, now in ((q, q2), (gq, g2)):
        lost = np.zeros((50, 96), bool)
        lost[7, 32:64] = True
        assert np.isnan(f64(now)[lost]).all() and (f64(now)[~lost] == f64(was)[~lost]).all()
