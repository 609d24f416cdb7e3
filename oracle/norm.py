"""Group norm with an activation over packed segments, channels last, its
gradients, and checkpoints in 8 bits: float64 numpy, one segment and group at a
time.  Test infrastructure; shares no code with the library.

    mean, var over the rows of a segment and the channels of a group,
    xn = (t - mean) / sqrt(var + eps), z = gamma xn + beta, y = act(z)
"""

import math

import numpy as np

IDENTITY, RELU, SILU, GELU = range(4)
BLOCK = 64

_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z, kind):
    if kind == RELU:
        return np.where(z > 0, z, 0.0)
    if kind == SILU:
        return z / (1.0 + np.exp(-z))
    if kind == GELU:
        return 0.5 * z * (1.0 + _erf(z / math.sqrt(2.0)))
    return z


def act_slope(z, kind):
    if kind == RELU:
        return (z > 0).astype(np.float64)
    if kind == SILU:
        p = 1.0 / (1.0 + np.exp(-z))
        return p + z * p * (1.0 - p)
    if kind == GELU:
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    return np.ones_like(z)


def bounds(n, segments):
    """The n_seg + 1 segment bounds: None (one), a count of equal ones, or the bounds themselves."""
    if segments is None:
        return np.array([0, n])
    if np.ndim(segments) == 0:
        return np.arange(segments + 1) * (n // segments)
    return np.asarray(segments)


def statistics(t, segments, groups, eps):
    """float64 [n_seg, groups, 2]: mean and rstd; zeros where a segment has no rows."""
    t = np.asarray(t, np.float64)
    n, C = t.shape
    b = bounds(n, segments)
    out = np.zeros((len(b) - 1, groups, 2))
    for s in range(len(b) - 1):
        if b[s + 1] > b[s]:
            v = t[b[s]:b[s + 1]].reshape(-1, groups, C // groups)
            mean = v.mean(axis=(0, 2))
            var = ((v - mean[None, :, None]) ** 2).mean(axis=(0, 2))
            out[s, :, 0], out[s, :, 1] = mean, 1.0 / np.sqrt(var + eps)
    return out


def normalised(t, stats, segments):
    """xn of every row."""
    t = np.asarray(t, np.float64)
    n, C = t.shape
    b = bounds(n, segments)
    row = np.repeat(np.arange(len(b) - 1), np.diff(b))
    c = C // stats.shape[1]
    mean, rstd = np.repeat(stats[row, :, 0], c, 1), np.repeat(stats[row, :, 1], c, 1)
    return (t - mean) * rstd


def forward(t, segments, groups, gamma, beta, kind, eps):
    """(y, stats)"""
    stats = statistics(t, segments, groups, eps)
    return act(normalised(t, stats, segments) * gamma + beta, kind), stats


def backward(t, stats, segments, gamma, beta, kind, grad_y):
    """(grad_t, dgamma, dbeta) with the given statistics of t."""
    t = np.asarray(t, np.float64)
    n, C = t.shape
    groups = stats.shape[1]
    c = C // groups
    b = bounds(n, segments)
    xn = normalised(t, stats, segments)
    w = np.asarray(grad_y, np.float64) * act_slope(xn * gamma + beta, kind)
    out = np.zeros((n, C))
    for s in range(len(b) - 1):
        r = slice(b[s], b[s + 1])
        if b[s + 1] == b[s]:
            continue
        gw, x = (w[r] * gamma).reshape(-1, groups, c), xn[r].reshape(-1, groups, c)
        A = gw.mean(axis=(0, 2))[None, :, None]
        B = (gw * x).mean(axis=(0, 2))[None, :, None]
        out[r] = (stats[s, :, 1][None, :, None] * (gw - A - x * B)).reshape(-1, C)
    return out, (w * xn).sum(0), w.sum(0)


def checkpoint(x):
    """(q int8, scale float32) of float32 rows, with the definition's own float32 steps."""
    x = np.asarray(x, np.float32)
    n, C = x.shape
    nb = -(-C // BLOCK)
    q = np.zeros((n, C), np.int8)
    scale = np.zeros((n, nb), np.float32)
    with np.errstate(all="ignore"):
        for k in range(nb):
            v = x[:, k * BLOCK:(k + 1) * BLOCK]
            a = np.abs(v).max(axis=1) if v.size else np.zeros(n, np.float32)
            odd = ~np.isfinite(v).all(axis=1)
            some = (a >= np.float32(2.0 ** -100)) & ~odd
            inv = np.where(some, np.float32(127.0) / a, np.float32(0)).astype(np.float32)
            scale[:, k] = np.where(odd, np.float32(np.nan), np.where(some, a * np.float32(1.0 / 127.0), np.float32(0)))
            t = np.where(some[:, None], np.rint(v * inv[:, None]), np.float32(0))
            q[:, k * BLOCK:(k + 1) * BLOCK] = np.clip(t, -127, 127).astype(np.int8)
    return q, scale


def values(q, scale):
    """The float32 values a checkpoint stands for."""
    C = q.shape[1]
    return q.astype(np.float32) * np.repeat(scale, BLOCK, axis=1)[:, :C]
