"""The attention layer's products in bfloat16: what it returns in float32 are float32 sums of the
products of its operands, not rounded on the way.

Tolerance: the products of two bfloat16 values are exact in float32, and K of them added in any
order are within K 2^-24 sum |a b| of the exact sum; 4 more for conversions."""

import numpy as np
import pytest

from tests.helpers import announce
from tests.test_gpu_attention_layer import Setup, env, f64  # noqa: F401

pytestmark = pytest.mark.gpu


class Watched:
    """The library, and the arguments and results of the layer's last attention and rotation calls."""

    def __init__(self, lib):
        self.lib, self.seen = lib, {}

    def __getattr__(self, name):
        call = getattr(self.lib, name)
        if not name.startswith("dsmp_"):
            return call

        def watched(*args, **kw):
            got = call(*args, **kw)
            self.seen[name] = (args, kw, got)
            return got

        return watched


def near(got, a, b):
    """got of float32 against the sums of a @ b in float64."""
    want, mag = a @ b, np.abs(a) @ np.abs(b)
    err = np.abs(f64(got) - want)
    assert str(got.dtype) == "torch.float32"
    assert (err <= (a.shape[1] + 4) * 2.0 ** -24 * mag).all(), float((err / np.maximum(mag, 1e-300)).max())


@pytest.mark.parametrize("kw", [dict(), dict(n=1500, H=8, Hk=2, hd=64, d=128, bounds=[0, 700, 1490])])
def test_results_are_float32_sums(env, kw):  # noqa: F811
    dm, lib, torch = env
    announce(kw)
    c = Setup(env, "bf16", **kw)
    c.gf = c.gf.bfloat16().float()
    seen = Watched(lib)
    layer = dm.AttentionLayer(seen, c.s)
    f = layer.forward(c.p, c.u, c.pos, c.seg)
    grad_u, grads = layer.backward(c.gf)
    torch.cuda.synchronize()
    p, u, gf = {k: f64(v) for k, v in c.p.items()}, f64(c.u), f64(c.gf)
    inside = np.zeros((c.s.n, 1))
    inside[c.bounds[0]:c.bounds[-1]] = 1.0
    out = f64(seen.seen["dsmp_attention_forward"][2][0])
    dq, dk, _ = seen.seen["dsmp_qk_rotate_backward"][2]
    dqkv = np.concatenate([f64(x) for x in (dq, dk, seen.seen["dsmp_attention_backward"][2][2])], 1)
    near(f, out, p["Wo"].T)
    near(grad_u, dqkv, p["Wqkv"])
    near(grads["dWqkv"], dqkv.T, u * inside)
    near(grads["dWo"], (gf * inside).T, out)


def test_reading_at_points_gives_float32_sums(env):  # noqa: F811
    dm, lib, torch = env
    c = Setup(env, "bf16", n=400)
    seen = Watched(lib)
    f = dm.AttentionLayer(seen, c.s).read(c.p, c.u[:7], c.pos[:7], c.u, c.pos)
    near(f, f64(seen.seen["dsmp_attention_forward"][2][0]), f64(c.p["Wo"]).T)
