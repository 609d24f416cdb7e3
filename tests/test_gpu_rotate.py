"""GPU parity of queries and keys normed and rotated in one pass, forward and backward,
against the float64 oracle.  Bounds, with u = 2^-24 and b half a step of the type:
  angle   the turns in float64, one turn rounded to float32: 2 pi u, and the sine's own 4 u
  u       (hd / 2 + 8) u |u|: squares added, a root, two products
  y       amp (|u_a| + |u_b|) (the angle's + 4 u) + the pair's bounds of u, + b |y|
  dx      r (the bound of w + |xn| that of the mean + (hd + 16) u of either), + b |dx|
  dgamma  sum |g xn| (the bounds of both + what adding them up in float32 loses) + u |dgamma|
"""

import numpy as np
import pytest

from oracle import attention as oa
from tests.helpers import announce, gpu_lib

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {"f32": U, "bf16": 2.0 ** -8 * 1.01}


@pytest.fixture(scope="module")
def env():
    return gpu_lib()


def f64(t):
    return t.detach().double().cpu().numpy()


class Case:
    def __init__(self, env, n, H, Hk, hd, dtype, rot, axes, layout, normed=True, amplitude=1.0, far=100.0, slices=False, seed=0):
        dm, lib, torch = env
        self.dm, self.lib, self.torch = dm, lib, torch
        self.n, self.hd, self.name, self.heads = n, hd, dtype, {"q": H, "k": Hk}
        self.dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        g = np.random.default_rng(seed + n + hd)
        cuda = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
        self.slices = slices
        self.x = {s: self.wide(cuda(2.0 * g.normal(size=(n, h * hd))).to(self.dt)) for s, h in self.heads.items()}
        self.dy = {s: self.wide(cuda(g.normal(size=(n, h * hd))).to(self.dt)) for s, h in self.heads.items()}
        self.gamma = {s: cuda(1 + 0.3 * g.normal(size=hd)) if normed else None for s in "qk"}
        self.pos = cuda(far * (2 * g.random((n, axes)) - 1))
        self.freq = dm.rotary_frequencies(rot, axes, device="cuda")
        self.rot, self.layout, self.amplitude, self.eps = rot, layout, amplitude, 1e-6 if normed else None
        self.desc = dm.rotate_desc(H, Hk, hd, {"f32": dm.F32, "bf16": dm.BF16}[dtype], rot, axes=axes, layout=layout,
                                   norm=normed, amplitude=amplitude)
        self.t = oa.angles(f64(self.pos), f64(self.freq), rot, axes)

    def wide(self, t):
        if not self.slices:
            return t
        w = self.torch.full((t.shape[0], t.shape[1] + 24), float("nan"), dtype=t.dtype, device=t.device)
        w[:, 16:16 + t.shape[1]] = t
        return w[:, 16:16 + t.shape[1]]

    def rows(self, t, s):
        return f64(t).reshape(self.n, self.heads[s], self.hd)

    def args(self):
        return self.gamma["q"], self.gamma["k"], self.pos, self.freq

    def turned_error(self, u, eu, sign=1.0):
        """Bound of the pairs of u turned, from u's own."""
        a, b = oa.pairs_of(self.rot, self.layout)
        e, amp = eu.copy(), abs(self.amplitude)
        both = (np.abs(u[:, :, a]) + np.abs(u[:, :, b])) * (2 * np.pi + 8) * U + eu[:, :, a] + eu[:, :, b]
        e[:, :, a] = e[:, :, b] = amp * both
        return e

    def check_forward(self, got, s):
        x = self.rows(self.x[s], s)
        gamma = None if self.gamma[s] is None else f64(self.gamma[s])
        want = oa.rotate(x, gamma, self.t, self.rot, self.layout, self.amplitude, self.eps)
        u = x if self.eps is None else oa.norm(x, self.eps)[0] * gamma
        eu = np.zeros_like(u) if self.eps is None else (self.hd / 2 + 8) * U * np.abs(u)
        tol = self.turned_error(u, eu) + HALF_STEP[self.name] * np.abs(want)
        err = np.abs(self.rows(got, s) - want)
        assert (err <= tol).all(), (s, float((err / np.maximum(tol, 1e-300)).max()))

    def check_backward(self, got, dgamma, s, before=0.0):
        x, dy = self.rows(self.x[s], s), self.rows(self.dy[s], s)
        gamma = None if self.gamma[s] is None else f64(self.gamma[s])
        want, want_g = oa.rotate_backward(x, gamma, self.t, self.rot, self.layout, self.amplitude, self.eps, dy)
        g = oa.turn(dy, self.t, self.rot, self.layout, self.amplitude, -1.0)
        eg = self.turned_error(dy, np.zeros_like(dy))
        tol = eg
        if self.eps is not None:
            xn, r = oa.norm(x, self.eps)
            n_u = (self.hd / 2 + 8) * U
            w, ew = g * gamma, np.abs(gamma) * (eg + 2 * U * np.abs(g))
            mag = (np.abs(w) * np.abs(xn)).mean(2, keepdims=True)
            em = (ew * np.abs(xn)).mean(2, keepdims=True) + (self.hd + 16) * U * mag + n_u * mag
            m = np.abs((w * xn).mean(2, keepdims=True))
            tol = r * (ew + np.abs(xn) * em + n_u * np.abs(xn) * m) + (n_u + 4 * U) * np.abs(want)
            tol = tol + 8 * U * r * (np.abs(w) + np.abs(xn) * m)
            count = self.n * self.heads[s]
            # at most 2 * 4 heads after one another in a lane's sum, 32 lanes, and the parts in float64: counted as one sum
            e_dg = ((eg + (n_u + 4 * U) * np.abs(g)) * np.abs(xn)).sum((0, 1)) + min(count, 4096) * U * (np.abs(g * xn)).sum((0, 1))
            e_dg = e_dg + 2 * U * (np.abs(want_g) + np.abs(before))
            assert (np.abs(f64(dgamma) - (want_g + before)) <= e_dg).all(), s
        tol = tol + HALF_STEP[self.name] * np.abs(want)
        err = np.abs(self.rows(got, s) - want)
        assert (err <= tol).all(), (s, float((err / np.maximum(tol, 1e-300)).max()))

    def check(self):
        q, k = self.lib.dsmp_qk_rotate_forward(self.desc, self.x["q"], self.x["k"], *self.args())
        self.torch.cuda.synchronize()
        self.check_forward(q, "q")
        self.check_forward(k, "k")
        gq, gk, dg = self.lib.dsmp_qk_rotate_backward(self.desc, self.x["q"], self.x["k"], *self.args(), self.dy["q"], self.dy["k"])
        self.torch.cuda.synchronize()
        self.check_backward(gq, dg.get("dgamma_q"), "q")
        self.check_backward(gk, dg.get("dgamma_k"), "k")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [oa.HALF, oa.INTERLEAVED])
@pytest.mark.parametrize("hd,rot,axes", [(8, 8, 1), (24, 6, 3), (32, 32, 2), (40, 24, 3), (64, 64, 1), (64, 0, 1), (72, 68, 2),
                                         (104, 20, 2), (128, 128, 2), (128, 96, 3)])
def test_widths_and_layouts(env, hd, rot, axes, layout, dtype):
    announce(dtype, layout, hd, rot, axes)
    Case(env, 37, 5, 2, hd, dtype, rot, axes, layout, slices=True).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,H,Hk", [(1, 8, 2), (3, 1, 1), (1000, 4, 4), (9001, 3, 16)])
def test_rows_and_heads(env, n, H, Hk, dtype):
    announce(dtype, n, H, Hk)
    Case(env, n, H, Hk, 32, dtype, 16, 2, oa.HALF, amplitude=1.25).check()


@pytest.mark.parametrize("layout", [oa.HALF, oa.INTERLEAVED])
@pytest.mark.parametrize("normed", [True, False])
def test_far_positions_keep_their_angles(env, layout, normed):
    """Whole-number positions up to 2^24: the angle has to be formed in more than 32 bits."""
    c = Case(env, 200, 2, 1, 64, "f32", 64, 1, layout, normed=normed, far=1.0)
    c.pos.copy_(c.torch.randint(2 ** 23, 2 ** 24, (200, 1)).float())
    c.t = oa.angles(f64(c.pos), f64(c.freq), c.rot, 1)
    c.check()


def test_one_of_both_and_in_place(env):
    dm, lib, torch = env
    c = Case(env, 300, 4, 2, 64, "bf16", 32, 1, oa.HALF)
    q, k = lib.dsmp_qk_rotate_forward(c.desc, c.x["q"], c.x["k"], *c.args())
    q1, none = lib.dsmp_qk_rotate_forward(c.desc, c.x["q"], None, c.gamma["q"], None, c.pos, c.freq)
    none2, k1 = lib.dsmp_qk_rotate_forward(c.desc, None, c.x["k"], None, c.gamma["k"], c.pos, c.freq)
    assert none is None and none2 is None and torch.equal(q, q1) and torch.equal(k, k1)
    gq, gk, dg = lib.dsmp_qk_rotate_backward(c.desc, c.x["q"], c.x["k"], *c.args(), c.dy["q"], c.dy["k"])
    g1, _, d1 = lib.dsmp_qk_rotate_backward(c.desc, c.x["q"], None, c.gamma["q"], None, c.pos, c.freq, c.dy["q"], None)
    c.check_backward(g1, d1["dgamma_q"], "q")
    assert torch.equal(g1, gq)
    d2 = c.dy["q"].clone(), c.dy["k"].clone()
    lib.dsmp_qk_rotate_backward(c.desc, c.x["q"], c.x["k"], *c.args(), *d2, grad_q=d2[0], grad_k=d2[1])
    x = c.x["q"].clone(), c.x["k"].clone()
    lib.dsmp_qk_rotate_forward(c.desc, *x, *c.args(), q_out=x[0], k_out=x[1])
    torch.cuda.synchronize()
    assert torch.equal(x[0], q) and torch.equal(x[1], k) and torch.equal(d2[0], gq) and torch.equal(d2[1], gk)


def test_one_gamma_and_accumulated_gradients(env):
    dm, lib, torch = env
    c = Case(env, 500, 4, 2, 32, "f32", 32, 1, oa.INTERLEAVED)
    before = torch.randn(32, device="cuda")
    grads = {"dgamma_q": before.clone()}
    c.gamma["k"] = None
    gq, gk, dg = lib.dsmp_qk_rotate_backward(c.desc, c.x["q"], c.x["k"], *c.args(), c.dy["q"], c.dy["k"], grads=grads,
                                             flags=dm.GRAD_ACCUMULATE)
    assert list(dg) == ["dgamma_q"]
    c.check_backward(gq, grads["dgamma_q"], "q", before=f64(before))
    none = torch.zeros(0, 128, device="cuda"), torch.zeros(0, 64, device="cuda")
    kept = grads["dgamma_q"].clone()
    lib.dsmp_qk_rotate_backward(c.desc, *none, c.gamma["q"], None, c.pos[:0], c.freq, *none, grads=grads, flags=dm.GRAD_ACCUMULATE)
    assert torch.equal(grads["dgamma_q"], kept)
    lib.dsmp_qk_rotate_backward(c.desc, *none, c.gamma["q"], None, c.pos[:0], c.freq, *none, grads=grads)
    assert not grads["dgamma_q"].any()


def test_same_on_every_run_and_replayed(env):
    dm, lib, torch = env
    c = Case(env, 5000, 4, 2, 64, "bf16", 64, 2, oa.HALF)
    size = lib.dsmp_qk_rotate_workspace(c.desc, c.n)

    def step(ws=None):
        q, k = lib.dsmp_qk_rotate_forward(c.desc, c.x["q"], c.x["k"], *c.args())
        gq, gk, dg = lib.dsmp_qk_rotate_backward(c.desc, c.x["q"], c.x["k"], *c.args(), c.dy["q"], c.dy["k"], ws=ws)
        return [q, k, gq, gk, dg["dgamma_q"], dg["dgamma_k"]]

    first = step()
    w = torch.full((size + 512,), 91, dtype=torch.uint8, device="cuda")
    assert all(torch.equal(x, y) for x, y in zip(step(w[256:256 + size]), first))
    torch.cuda.synchronize()
    assert (w[:256] == 91).all() and (w[-256:] == 91).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        held = step()
    for i in range(3):
        c.x["q"].mul_(1.5)
        c.dy["k"].add_(0.25)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want))


def test_refusals(env):
    dm, lib, torch = env
    c = Case(env, 8, 2, 1, 32, "bf16", 32, 1, oa.HALF)

    def refused(status, desc=c.desc, q=c.x["q"], k=c.x["k"], gq=c.gamma["q"], gk=c.gamma["k"], pos=c.pos, freq=c.freq):
        with pytest.raises(dm.DsmpError) as e:
            lib.dsmp_qk_rotate_forward(desc, q, k, gq, gk, pos, freq)
        assert e.value.status == status, e.value

    bad = dm.INVALID_ARG
    refused(bad, q=None, k=None)
    refused(bad, q=c.x["q"].float())
    refused(bad, q=c.x["q"][:4])
    refused(bad, pos=None)
    refused(bad, freq=c.freq[:3])
    refused(bad, gq=c.gamma["q"][:8])
    refused(bad, desc=dm.rotate_desc(2, 1, 32, dm.BF16, 32, norm=False))            # gammas without a norm
    refused(bad, desc=dm.rotate_desc(2, 1, 32, dm.BF16, 30, axes=2), freq=c.freq[:15], pos=torch.zeros(8, 2, device="cuda"))
    refused(bad, q=torch.zeros(8, 68, dtype=torch.bfloat16, device="cuda")[:, :64])
    refused(bad, desc=dm.rotate_desc(2, 1, 32, dm.BF16, 32, layout=2))
