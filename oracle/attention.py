"""Queries and keys normed and rotated, and attention within packed segments, with
their gradients: float64 numpy, one segment and head at a time.  Test
infrastructure; shares no code with the library.

    u = gamma x / sqrt(mean x^2 + eps), pairs turned by pos[axis] * freq
    z = c(scale q.k) - slope |p_i - p_j|, c(x) = cap tanh(x / cap)
    out = softmax(z) v, lse = log sum e^z

``attention`` and ``attention_backward`` return, beside each result, an elementwise
bound of what roundings may change it by (see ``Errors``).
"""

import numpy as np

HALF, INTERLEAVED = 0, 1
U = 2.0 ** -24
# float32 results below this may be 0 instead (the hardware's powers have no subnormal results): weights
# e^(z - lse) of keys that score 88 below the row's sum, and products with them
TINY = 2.0 ** -126


def pairs_of(rot, layout):
    p = np.arange(rot // 2)
    return (p, p + rot // 2) if layout == HALF else (2 * p, 2 * p + 1)


def angles(pos, freq, rot, axes):
    """float64 [n, rot / 2]"""
    half = rot // 2
    axis = np.arange(half) * axes // max(half, 1)
    return np.asarray(pos, np.float64)[:, axis] * np.asarray(freq, np.float64)


def turn(u, t, rot, layout, amplitude, sign=1.0):
    """Rows [n, heads, hd] with their pairs turned by t (sign -1: back)."""
    a, b = pairs_of(rot, layout)
    y = u.copy()
    c, s = np.cos(t)[:, None], sign * np.sin(t)[:, None]
    y[:, :, a] = amplitude * (u[:, :, a] * c - u[:, :, b] * s)
    y[:, :, b] = amplitude * (u[:, :, a] * s + u[:, :, b] * c)
    return y


def norm(x, eps):
    """(x / rms, 1 / rms)"""
    r = 1.0 / np.sqrt((x * x).mean(2, keepdims=True) + eps)
    return x * r, r


def rotate(x, gamma, t, rot, layout, amplitude, eps):
    """x float64 [n, heads, hd]; gamma and eps None: not normed."""
    u = x if eps is None else norm(x, eps)[0]
    return turn(u if gamma is None else u * gamma, t, rot, layout, amplitude)


def rotate_backward(x, gamma, t, rot, layout, amplitude, eps, dy):
    """(dx, dgamma)"""
    g = turn(dy, t, rot, layout, amplitude, -1.0)
    if eps is None:
        return g, None
    xn, r = norm(x, eps)
    w = g if gamma is None else g * gamma
    return r * (w - xn * (w * xn).mean(2, keepdims=True)), (g * xn).sum((0, 1))


class Errors:
    """What float32 (and, in products, `half`) arithmetic may change results by.

    half: half a step of the type of the products' operands, relative (2^-8 for
    bfloat16, 2^-24 for float32), which P, the scores' gradients and the results are
    rounded to.  cap_abs: absolute error of tanh."""

    def __init__(self, half, cap_abs):
        self.half, self.cap_abs = half, cap_abs

    def score(self, qk, x, z, bias, hd, scale, cap):
        """Of z: hd products added in float32 (their magnitudes qk), a scale, the bias
        (differences, squares, a root and a product: 8 u), and the conversion to powers of
        two and back (4 u of each term)."""
        e = (hd + 4) * U * abs(scale) * qk + 8 * U * (np.abs(x) + np.abs(z) + bias)
        return e + (cap * (self.cap_abs + 4 * U) if cap else 0.0)


def _segments(bounds):
    return [slice(int(a), int(b)) for a, b in zip(bounds, bounds[1:])]


def _scores(q, k, pos_q, pos_k, slope, scale, cap, err):
    qk, mag = q @ k.T, np.abs(q) @ np.abs(k).T
    x = scale * qk
    t = np.tanh(x / cap) if cap else None
    z, bias = (cap * t if cap else x), np.zeros_like(x)
    if pos_q is not None:
        d = pos_q[:, None].astype(np.float64) - pos_k[None].astype(np.float64)
        bias = slope * np.sqrt((d * d).sum(2))
        z = z - bias
    fall = 1.0 - t * t if cap else np.ones_like(x)
    return z, fall, err.score(mag, x, z, np.abs(bias), q.shape[1], scale, cap)


def attention(q, k, v, q_bounds, k_bounds, scale, cap=0.0, pos_q=None, pos_k=None, slopes=None, err=Errors(U, 0.0)):
    """q [nq, H, hd], k, v [nk, Hk, hd] float64; returns out, lse and their bounds.  Rows of no
    segment are NaN."""
    H, G = q.shape[1], q.shape[1] // k.shape[1]
    out, lse = np.full_like(q, np.nan), np.full((q.shape[0], H), np.nan)
    e_out, e_lse = np.zeros_like(q), np.zeros_like(lse)
    for a, b in zip(_segments(q_bounds), _segments(k_bounds)):
        n = b.stop - b.start
        for h in range(H):
            if n <= 0:
                out[a, h], lse[a, h] = 0.0, -np.inf
                continue
            args = (None, None, 0.0) if pos_q is None else (pos_q[a], pos_k[b], float(slopes[h]))
            z, _, ez = _scores(q[a, h], k[b, h // G], *args, scale, cap, err)
            top = z.max(1, keepdims=True)
            lse[a, h] = (top + np.log(np.exp(z - top).sum(1, keepdims=True)))[:, 0]
            P = np.exp(z - lse[a, h][:, None])
            out[a, h] = P @ v[b, h // G]
            ez = ez.max(1, keepdims=True)
            # a weight and the sum of weights: the score's error, the power's and its argument's difference (8 u of
            # it is in the score's), n additions each in numerator and sum, joined parts
            rel = 2 * ez + (2 * n + 32) * U + err.half
            e_out[a, h] = rel * (P @ np.abs(v[b, h // G])) + TINY * np.abs(v[b, h // G]).sum(0) + 1.01 * err.half * np.abs(out[a, h])
            e_lse[a, h] = (ez + (n + 32) * U)[:, 0] + 4 * U * np.abs(lse[a, h]) + 4 * U
    return out, lse, e_out, e_lse


def attention_backward(q, k, v, do, q_bounds, k_bounds, scale, cap=0.0, pos_q=None, pos_k=None, slopes=None,
                       err=Errors(U, 0.0)):
    """(dq, dk, dv) and their bounds, for the exact forward results.  Keys of segments without
    queries have zeros, rows of no segment NaN."""
    H, hd, G = q.shape[1], q.shape[2], q.shape[1] // k.shape[1]
    out, lse, e_out, e_lse = attention(q, k, v, q_bounds, k_bounds, scale, cap, pos_q, pos_k, slopes, err)
    dq, dk, dv = np.full_like(q, np.nan), np.full_like(k, np.nan), np.full_like(v, np.nan)
    eq, ek, ev = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for a, b in zip(_segments(q_bounds), _segments(k_bounds)):
        n, m = b.stop - b.start, (a.stop - a.start) * G
        dq[a], dk[b], dv[b] = 0.0, 0.0, 0.0
        if n <= 0 or m <= 0:
            continue
        for h in range(H):
            j = h // G
            Q, K, V, g, o = q[a, h], k[b, j], v[b, j], do[a, h], out[a, h]
            args = (None, None, 0.0) if pos_q is None else (pos_q[a], pos_k[b], float(slopes[h]))
            z, fall, ez = _scores(Q, K, *args, scale, cap, err)
            P = np.exp(z - lse[a, h][:, None])
            dP, D = g @ V.T, (g * o).sum(1, keepdims=True)
            dS = P * (dP - D) * fall
            eP = ez + e_lse[a, h][:, None] + 16 * U
            e_dP = (hd + 4) * U * (np.abs(g) @ np.abs(V).T)
            e_D = (np.abs(g) * e_out[a, h]).sum(1, keepdims=True) + (hd + 4) * U * (np.abs(g) * np.abs(o)).sum(1, keepdims=True)
            e_fall = (4 * err.cap_abs + 8 * U + 2 * ez / cap) if cap else 0.0
            e_dS = np.abs(dS) * (eP + 8 * U + err.half) + P * fall * (e_dP + e_D) + P * np.abs(dP - D) * e_fall
            e_dS = e_dS + TINY * (1.0 + np.abs(dP - D))
            dv[b, j] += P.T @ g
            ev[b, j] += (P * (eP + err.half + (m + 16) * U) + 2 * TINY).T @ np.abs(g)
            dq[a, h] = scale * (dS @ K)
            eq[a, h] = abs(scale) * (e_dS + (n + 16) * U * np.abs(dS)) @ np.abs(K)
            dk[b, j] += scale * (dS.T @ Q)
            ek[b, j] += abs(scale) * (e_dS + (m + 16) * U * np.abs(dS)).T @ np.abs(Q)
    with np.errstate(invalid="ignore"):
        return dq, dk, dv, *(e + 1.01 * err.half * np.abs(x) for e, x in ((eq, dq), (ek, dk), (ev, dv)))
