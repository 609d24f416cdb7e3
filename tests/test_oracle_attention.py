"""The attention oracle against differences and against cases worked out by hand."""

import numpy as np
import pytest

from oracle import attention as oa


def _case(seed, nq, nk, H, Hk, hd, dim):
    g = np.random.default_rng(seed)
    q, k, v, do = (g.normal(size=s) for s in ((nq, H, hd), (nk, Hk, hd), (nk, Hk, hd), (nq, H, hd)))
    at = (None, None, None) if not dim else (g.random((nq, dim)), g.random((nk, dim)), 4 * g.random(H))
    return q, k, v, do, at


@pytest.mark.parametrize("cap,dim", [(0.0, 0), (2.0, 0), (0.0, 2), (3.0, 3)])
def test_gradients_match_differences(cap, dim):
    q, k, v, do, at = _case(1, 5, 7, 4, 2, 8, dim)
    qb, kb, scale = [0, 2, 2, 5], [0, 4, 6, 7], 0.4

    def loss(q, k, v):
        return float((oa.attention(q, k, v, qb, kb, scale, cap, *at)[0] * do).sum())

    grads = oa.attention_backward(q, k, v, do, qb, kb, scale, cap, *at)[:3]
    rng = np.random.default_rng(2)
    for which, g in enumerate(grads):
        for _ in range(3):
            d = rng.normal(size=g.shape)
            args = [[x.copy() for x in (q, k, v)] for _ in range(2)]
            args[0][which] += 1e-5 * d
            args[1][which] -= 1e-5 * d
            diff = (loss(*args[0]) - loss(*args[1])) / 2e-5
            # central differences: third derivatives times 1e-10, and 1e-16 of the loss over the step
            assert abs(diff - (g * d).sum()) <= 1e-7 * (1 + abs(diff))


def test_uniform_scores_average_the_values_and_segments_do_not_mix():
    v = np.arange(12.0).reshape(6, 1, 2)
    k, q = np.zeros((6, 1, 2)), np.ones((3, 1, 2))
    v[4:] = np.nan                                            # of the second segment, which has no queries
    out, lse, _, _ = oa.attention(q, k, v, [0, 2, 2, 3], [0, 4, 6, 6], 1.0)
    assert np.array_equal(out[:2, 0], np.tile(v[:4, 0].mean(0), (2, 1))) and np.allclose(lse[:2], np.log(4.0), rtol=1e-15)
    assert np.array_equal(out[2], np.zeros((1, 2))) and lse[2, 0] == -np.inf


def test_a_distance_of_three_and_four_is_five():
    q = k = np.zeros((1, 1, 2))
    _, lse, _, _ = oa.attention(q, k, k, [0, 1], [0, 1], 1.0, 0.0, np.array([[0.0, 3.0]]), np.array([[4.0, 0.0]]), [2.0])
    assert lse[0, 0] == -10.0


@pytest.mark.parametrize("layout", [oa.HALF, oa.INTERLEAVED])
def test_rotation_by_hand_and_its_gradient(layout):
    x = np.arange(1.0, 9.0).reshape(1, 1, 8)
    t = oa.angles(np.array([[np.pi / 2, 0.0]]), np.array([1.0, 1.0]), 4, 2)
    y = oa.rotate(x, None, t, 4, layout, 2.0, None)[0, 0]
    want = [-6, 4, 2, 8] if layout == oa.HALF else [-4, 2, 6, 8]   # the first pair a quarter turn, the second none
    assert np.allclose(y, want + [5, 6, 7, 8], atol=1e-14)
    g = np.random.default_rng(3)
    x, dy, gamma = g.normal(size=(3, 2, 8)), g.normal(size=(3, 2, 8)), 1 + 0.1 * g.normal(size=8)
    t = g.normal(size=(3, 3))

    def loss(x, gamma):
        return float((oa.rotate(x, gamma, t, 6, layout, 1.3, 1e-3) * dy).sum())

    dx, dgamma = oa.rotate_backward(x, gamma, t, 6, layout, 1.3, 1e-3, dy)
    d, e = g.normal(size=x.shape), g.normal(size=8)
    assert abs((loss(x + 1e-5 * d, gamma) - loss(x - 1e-5 * d, gamma)) / 2e-5 - (dx * d).sum()) <= 1e-7
    assert abs((loss(x, gamma + 1e-5 * e) - loss(x, gamma - 1e-5 * e)) / 2e-5 - (dgamma * e).sum()) <= 1e-7
