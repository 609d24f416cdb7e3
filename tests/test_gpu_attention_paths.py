"""GPU parity of attention on every kind of tile, whole and cut (see ``attention_paths``), against the
float64 oracle within its bounds: all heads where their scores are few, else a key head here and there."""

import numpy as np
import pytest

from oracle import attention as oa
from tests.attention_paths import PATHS, bounds
from tests.helpers import announce
from tests.test_gpu_attention import Case, env, f64  # noqa: F401

pytestmark = pytest.mark.gpu

# half a step of the type; tanh: in float32 the kernels' own, within 3 units of 2^-24, in bfloat16 from the hardware's power and
# reciprocal, within 2^-22 of 1 - 2 / (1 + e^2x)
ERRORS = {"f32": oa.Errors(2.0 ** -24, 3 * 2.0 ** -24), "bf16": oa.Errors(2.0 ** -8, 2.0 ** -21)}
SCORES = 4e6   # that the oracle forms for one call


@pytest.mark.parametrize("i", range(len(PATHS)))
def test_tiles(env, i):  # noqa: F811
    dtype, hd, dim, cap, Hk, G, what, room, plan = PATHS[i]
    announce(*PATHS[i])
    qb, kb = bounds(what)
    c = Case(env, qb, kb, Hk * G, Hk, hd, dtype, dim=dim, cap=cap, room=room, slices=i % 3 == 0)
    torch = c.torch
    out, lse = c.forward()
    grads = c.backward(out, lse)
    torch.cuda.synchronize()
    for t, b in ((out, qb), (lse, qb), (grads[0], qb), (grads[1], kb), (grads[2], kb)):
        assert (t[:b[0]] == 77.0).all() and (t[b[-1]:] == 77.0).all(), "rows of no segment"
        assert not t[b[0]:b[-1]].isnan().any()
    scores = G * sum((q1 - q0) * (k1 - k0) for q0, q1, k0, k1 in zip(qb, qb[1:], kb, kb[1:]))
    some = max(1, min(Hk, int(SCORES / scores)))
    of = [Hk - 1] if some == 1 else sorted({j * (Hk - 1) // (some - 1) for j in range(some)})
    heads = [j * G + g for j in of for g in range(G)]
    a, b = slice(qb[0], qb[-1]), slice(kb[0], kb[-1])
    # rows of the segments alone
    rows = lambda t, s, which, H: f64(t[s]).reshape(s.stop - s.start, H, hd)[:, which]  # noqa: E731
    q, do, k, v = rows(c.q, a, heads, Hk * G), rows(c.do, a, heads, Hk * G), rows(c.k, b, of, Hk), rows(c.v, b, of, Hk)
    place = (None, None, None)
    if dim:
        pos, k_pos, slopes = c.places()
        place = pos[a], k_pos[b], slopes[heads]
    args = ([x - qb[0] for x in qb], [x - kb[0] for x in kb], c.scale, cap, *place)
    w_out, w_lse, e_out, e_lse = oa.attention(q, k, v, *args, err=ERRORS[dtype])
    want = oa.attention_backward(q, k, v, do, *args, err=ERRORS[dtype])
    got = dict(out=(rows(out, a, heads, Hk * G), w_out, e_out), lse=(f64(lse[a])[:, heads], w_lse, e_lse),
               dq=(rows(grads[0], a, heads, Hk * G), want[0], want[3]), dk=(rows(grads[1], b, of, Hk), want[1], want[4]),
               dv=(rows(grads[2], b, of, Hk), want[2], want[5]))
    for name, (g, w, tol) in got.items():
        with np.errstate(invalid="ignore"):
            far = np.where(g == w, 0.0, np.abs(g - w) / np.maximum(tol, 1e-300))     # equal: infinities of rows without keys
        assert (far <= 1.0).all(), (name, float(far.max()))
    # the same on every run
    again = c.forward()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    assert all(torch.equal(x, y) for x, y in zip(c.backward(out, lse), grads))
