"""Pins of the norm and checkpoint oracle (CPU): hand-worked values, closed
forms, invariances, central differences of every gradient, the checkpoint's
error bound and its special blocks."""

import math

import numpy as np
import pytest

from oracle import norm as on


def test_hand_worked_segment():
    # two segments of two rows, one group of two channels; the first holds 1, 3, 5, 7
    t = np.array([[1.0, 3.0], [5.0, 7.0], [2.0, 2.0], [2.0, 2.0]])
    y, st = on.forward(t, [0, 2, 4], 1, np.array([2.0, 1.0]), np.array([0.0, 1.0]), on.IDENTITY, 0.25)
    assert st[0, 0, 0] == 4.0 and st[1, 0, 0] == 2.0
    assert st[0, 0, 1] == pytest.approx(1 / math.sqrt(5.25)) and st[1, 0, 1] == 2.0
    r = 1 / math.sqrt(5.25)
    np.testing.assert_allclose(y, [[-6 * r, 1 - r], [2 * r, 1 + 3 * r], [0, 1], [0, 1]], rtol=1e-15)


def test_activations_at_known_points():
    z = np.array([-1.0, 0.0, 2.0])
    np.testing.assert_allclose(on.act(z, on.RELU), [0, 0, 2])
    np.testing.assert_allclose(on.act(z, on.SILU), [-1 / (1 + math.e), 0, 2 / (1 + math.exp(-2))], rtol=1e-15)
    np.testing.assert_allclose(on.act(z, on.GELU), [-0.15865525393145707, 0, 1.9544997361036416], rtol=1e-13)
    assert on.act_slope(np.array([0.0]), on.RELU)[0] == 0.0


@pytest.mark.parametrize("segments", [None, 4, [0, 0, 3, 3, 11, 12, 12]])
def test_segments_are_independent_and_normalised(segments):
    g = np.random.default_rng(0)
    t = g.normal(size=(12, 6)) * 3 + 1
    y, st = on.forward(t, segments, 2, np.ones(6), np.zeros(6), on.IDENTITY, 0.0)
    b = on.bounds(12, segments)
    for s in range(len(b) - 1):
        v = y[b[s]:b[s + 1]].reshape(-1, 2, 3)
        if len(v) == 0:
            assert (st[s] == 0).all()
            continue
        np.testing.assert_allclose(v.mean(axis=(0, 2)), 0, atol=1e-12)
        np.testing.assert_allclose((v ** 2).mean(axis=(0, 2)), 1, rtol=1e-12)
        alone, _ = on.forward(t[b[s]:b[s + 1]], None, 2, np.ones(6), np.zeros(6), on.IDENTITY, 0.0)
        np.testing.assert_allclose(alone, y[b[s]:b[s + 1]], rtol=1e-12, atol=1e-14)


@pytest.mark.parametrize("kind", [on.IDENTITY, on.RELU, on.SILU, on.GELU])
@pytest.mark.parametrize("segments", [None, [0, 1, 1, 5, 9], 9])
def test_gradients_against_central_differences(kind, segments):
    g = np.random.default_rng(kind + 10)
    n, C, groups, eps, h = 9, 8, 2, 0.1, 1e-5
    t, dy = g.normal(size=(n, C)) * 2 + 1, g.normal(size=(n, C))
    P = {"t": t, "gamma": 1 + 0.3 * g.normal(size=C), "beta": 0.3 * g.normal(size=C)}

    def loss(p):
        return float((on.forward(p["t"], segments, groups, p["gamma"], p["beta"], kind, eps)[0] * dy).sum())

    stats = on.statistics(t, segments, groups, eps)
    z = on.normalised(t, stats, segments) * P["gamma"] + P["beta"]
    assert kind != on.RELU or np.abs(z).min() > 1e-3      # no kink within a step
    got = dict(zip(("t", "gamma", "beta"), on.backward(t, stats, segments, P["gamma"], P["beta"], kind, dy)))
    for name, v in P.items():
        for i in np.ndindex(v.shape):
            up, dn = dict(P), dict(P)
            up[name], dn[name] = v.copy(), v.copy()
            up[name][i] += h
            dn[name][i] -= h
            assert got[name][i] == pytest.approx((loss(up) - loss(dn)) / (2 * h), abs=2e-8, rel=1e-6), (name, i)


@pytest.mark.parametrize("C", [1, 5, 64, 65, 200])
def test_checkpoint_error_is_at_most_half_a_step(C):
    g = np.random.default_rng(C)
    x = (g.normal(size=(50, C)) * np.exp(3 * g.normal(size=(50, 1)))).astype(np.float32)
    q, scale = on.checkpoint(x)
    v = on.values(q, scale)
    step = np.repeat(scale, on.BLOCK, 1)[:, :C].astype(np.float64)
    assert (np.abs(v.astype(np.float64) - x) <= step * (0.5 + 2.0 ** -15)).all()
    # the largest of a block keeps its value up to rounding
    for k in range(scale.shape[1]):
        b = slice(64 * k, min(C, 64 * (k + 1)))
        np.testing.assert_allclose(np.abs(v[:, b]).max(1), np.abs(x[:, b]).max(1), rtol=3e-7)


def test_checkpoint_of_special_blocks():
    x = np.zeros((5, 70), np.float32)
    x[1, 3], x[1, 69] = np.inf, 2.0
    x[2, 5], x[2, 69] = np.nan, -2.0
    x[3, 0] = 2.0 ** -101
    x[4, :2] = [127.0, 2.5]
    q, scale = on.checkpoint(x)
    v = on.values(q, scale)
    assert (v[0] == 0).all() and (v[3] == 0).all()
    assert np.isnan(v[1, :64]).all() and np.isnan(v[2, :64]).all() and (q[1:3, :64] == 0).all()
    assert q[1, 69] == 127 and q[2, 69] == -127 and np.isfinite(v[1:3, 64:]).all()
    assert q[4, 0] == 127 and q[4, 1] == 2          # 2.5 goes to the even neighbour
