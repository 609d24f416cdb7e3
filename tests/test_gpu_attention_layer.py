"""The attention layer (norm, projections, rotation, attention, projection) as a training
step runs it, forward and backward, between group norms and a message-passing layer, against
the float64 oracle's pieces; its evaluation at a few points; a captured step.

Parity as for the message-passing layers: the largest difference over the largest value,
1e-4 in float32 and 2e-2 in bfloat16."""

import numpy as np
import pytest

from oracle import attention as oa
from tests.helpers import TOL, announce, gpu_lib, rel_err

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    return gpu_lib()


def f64(t):
    return t.detach().double().cpu().numpy()


class Setup:
    def __init__(self, env, dtype, n=300, bounds=None, d=64, H=4, Hk=2, hd=32, dim=2, cap=5.0, seed=0, **kw):
        dm, lib, torch = env
        self.dm, self.lib, self.torch, self.name = dm, lib, torch, dtype
        self.dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.s = dm.AttentionShapes(n=n, d=d, heads=H, kv_heads=Hk, head_dim=hd, dtype={"f32": dm.F32, "bf16": dm.BF16}[dtype],
                                    dim=dim, rot=kw.get("rot", hd), layout=kw.get("layout", dm.ROTATE_HALF), cap=cap,
                                    norm=kw.get("norm", True), distance=kw.get("distance", True))
        g = np.random.default_rng(seed)
        cuda = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
        self.p = {"Wqkv": cuda(g.normal(size=((H + 2 * Hk) * hd, d)) / d ** 0.5).to(self.dt),
                  "Wo": cuda(g.normal(size=(d, H * hd)) / (H * hd) ** 0.5).to(self.dt),
                  "freq": dm.rotary_frequencies(self.s.rot, dim, base=100.0, device="cuda"), "slopes": cuda(3 * g.random(H))}
        if self.s.norm:
            self.p.update(gamma_q=cuda(1 + 0.2 * g.normal(size=hd)), gamma_k=cuda(1 + 0.2 * g.normal(size=hd)))
        self.u = cuda(g.normal(size=(n, d))).to(self.dt)
        self.pos, self.gf = cuda(3 * g.random((n, dim))), cuda(g.normal(size=(n, d)))
        self.bounds = bounds or [0, n]
        self.seg = torch.tensor(bounds, dtype=torch.int32, device="cuda") if bounds else None

    def reference(self, u, gf, uk=None, pos=None, k_pos=None, qb=None, kb=None):
        """(f, grad_u, grads) in float64; f alone for other points than the nodes."""
        s, p = self.s, {k: f64(v) for k, v in self.p.items()}
        wq, wk = s.heads * s.head_dim, s.kv_heads * s.head_dim
        pos = f64(self.pos) if pos is None else pos
        k_pos, uk = (pos, u) if k_pos is None else (k_pos, uk)
        qb, kb = qb or self.bounds, kb or self.bounds
        W = p["Wqkv"]
        heads = lambda x, H: x.reshape(len(x), H, s.head_dim)  # noqa: E731
        q, k, v = heads(u @ W[:wq].T, s.heads), heads(uk @ W[wq:wq + wk].T, s.kv_heads), heads(uk @ W[wq + wk:].T, s.kv_heads)
        eps, gq, gk = (s.eps, p["gamma_q"], p["gamma_k"]) if s.norm else (None, None, None)
        tq, tk = oa.angles(pos, p["freq"], s.rot, s.dim), oa.angles(k_pos, p["freq"], s.rot, s.dim)
        qr, kr = oa.rotate(q, gq, tq, s.rot, s.layout, 1.0, eps), oa.rotate(k, gk, tk, s.rot, s.layout, 1.0, eps)
        at = (pos, k_pos, p["slopes"]) if s.distance else (None, None, None)
        args = (qb, kb, s.head_dim ** -0.5, s.cap, *at)
        out = np.nan_to_num(oa.attention(qr, kr, v, *args)[0]).reshape(len(u), wq)
        f = out @ p["Wo"].T
        if gf is None:
            return f
        dout = heads(gf @ p["Wo"], s.heads)
        dqr, dkr, dv = (np.nan_to_num(x) for x in oa.attention_backward(qr, kr, v, dout, *args)[:3])
        dq, dgq = oa.rotate_backward(q, gq, tq, s.rot, s.layout, 1.0, eps, dqr)
        dk, dgk = oa.rotate_backward(k, gk, tk, s.rot, s.layout, 1.0, eps, dkr)
        dqkv = np.concatenate([x.reshape(len(u), -1) for x in (dq, dk, dv)], 1)
        grads = {"dWqkv": dqkv.T @ u, "dWo": gf.T @ out}
        if s.norm:
            grads.update(dgamma_q=dgq, dgamma_k=dgk)
        return f, dqkv @ W, grads

    def check(self):
        layer = self.dm.AttentionLayer(self.lib, self.s)
        f = layer.forward(self.p, self.u, self.pos, self.seg)
        grad_u, grads = layer.backward(self.gf)
        self.torch.cuda.synchronize()
        inside = np.zeros((self.s.n, 1), bool)
        inside[self.bounds[0]:self.bounds[-1]] = True
        w_f, w_u, w_g = self.reference(f64(self.u), f64(self.gf))
        tol = TOL[self.name]
        assert rel_err(f64(f), w_f) <= tol
        assert rel_err(f64(grad_u), w_u) <= tol
        assert set(grads) == set(w_g)
        for name, w in w_g.items():
            assert rel_err(f64(grads[name]), w) <= tol, name
        assert not f64(f)[~inside[:, 0]].any() and not f64(grad_u)[~inside[:, 0]].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(), dict(bounds=[0, 70, 70, 200, 290]), dict(H=2, Hk=2, hd=40, rot=24, dim=3, cap=0.0, layout=1),
                                dict(norm=False, distance=False, rot=0, cap=0.0), dict(n=1500, H=8, Hk=1, hd=64, bounds=[0, 700, 1500])])
def test_layer(env, kw, dtype):
    announce(dtype, kw)
    Setup(env, dtype, **kw).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_read_at_points(env, dtype):
    """Seven points in three sub-domains read the field of their nodes."""
    c = Setup(env, dtype, n=400, bounds=[0, 150, 151, 400])
    torch = c.torch
    g = np.random.default_rng(9)
    u = torch.tensor(g.normal(size=(7, c.s.d)), dtype=torch.float32, device="cuda").to(c.dt)
    pos = torch.tensor(3 * g.random((7, c.s.dim)), dtype=torch.float32, device="cuda")
    qb = [0, 3, 4, 7]
    layer = c.dm.AttentionLayer(c.lib, c.s)
    f = layer.read(c.p, u, pos, c.u, c.pos, torch.tensor(qb, dtype=torch.int32, device="cuda"), c.seg)
    want = c.reference(f64(u), None, f64(c.u), f64(pos), f64(c.pos), qb, c.bounds)
    assert rel_err(f64(f), want) <= TOL[dtype]


def test_between_norms_and_message_passing(env):
    """A block as a stack runs it: norm, attention, the sum and the next norm in one call, a
    message-passing layer; its gradient along a direction against differences (float32)."""
    dm, lib, torch = env
    c = Setup(env, "f32", n=256, d=32, H=2, Hk=1, hd=32, cap=0.0)
    n, d = 256, 32
    graph = lib.dsmp_radius_graph_build(c.pos, n, 0.4)
    conv = dm.layer_desc(2, d, 64, 64, dm.F32, dm.ACT_IDENTITY, 0, dm.ATTR_CONCAT)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    rnd = lambda *s: (2 * torch.rand(*s, generator=gen, device="cuda") - 1) * s[-1] ** -0.5  # noqa: E731
    packed = lib.dsmp_nnconv_pack(conv, {"W1": rnd(64, 6), "b1": rnd(64), "W2": rnd(64, 64), "b2": rnd(64), "W3": rnd(d * d, 64),
                                         "b3": rnd(d * d), "Wr": rnd(d, d), "br": rnd(d)})
    attr = torch.cat([c.pos, torch.randn(n, 1, generator=gen, device="cuda")], 1)
    desc = dm.norm_desc(d, 4, dm.F32, dm.F32)
    one, zero = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
    layer = dm.AttentionLayer(lib, c.s)
    gy = torch.randn(n, d, generator=gen, device="cuda")

    def forward(x):
        u, st1 = lib.dsmp_group_norm_forward(desc, x, one, zero)
        f = layer.forward(c.p, u, c.pos)
        total = torch.empty_like(x)
        w, st2 = lib.dsmp_group_norm_forward(desc, x, one, zero, addend=f, sum_out=total)
        y, saved = lib.dsmp_nnconv_forward(conv, packed, graph, attr, w)
        return y, (st1, total, w, st2, saved)

    x = torch.randn(n, d, generator=gen, device="cuda")
    y, (st1, total, w, st2, saved) = forward(x)
    gw, _ = lib.dsmp_nnconv_backward(conv, packed, graph, attr, w, saved, gy)
    gt, _ = lib.dsmp_group_norm_backward(desc, total, st2, one, zero, gw)
    gu, _ = layer.backward(gt)
    gx, _ = lib.dsmp_group_norm_backward(desc, x, st1, one, zero, gu, grad_addend=gt)
    v = torch.randn(n, d, generator=gen, device="cuda")
    loss = lambda t: float((forward(t)[0].double() * gy.double()).sum())  # noqa: E731
    h = 2.0 ** -7
    d1, d2 = ((loss(x + k * v) - loss(x - k * v)) / (2 * k) for k in (h, h / 2))
    want = float((gx.double() * v.double()).sum())
    # each y is within 1e-4 of the largest (the parity of the calls), the sum of 8,192 of them over h / 2
    noise = 1e-4 * float(y.abs().max()) * float(gy.norm()) / h
    assert abs((4 * d2 - d1) / 3 - want) <= noise + abs(d2 - d1), (d1, d2, want)


def test_captured_step_and_refusals(env):
    dm, lib, torch = env
    c = Setup(env, "bf16", n=500)
    layer = dm.AttentionLayer(lib, c.s)
    with pytest.raises(dm.DsmpError):
        layer.backward(c.gf)
    with pytest.raises(dm.DsmpError):
        layer.forward(c.p, c.u[:10], c.pos)
    with pytest.raises(dm.DsmpError):
        layer.forward(c.p, c.u.float(), c.pos)
    with pytest.raises(dm.DsmpError):
        layer.backward(c.gf)                      # none of them came to its end

    def step():
        f = layer.forward(c.p, c.u, c.pos)
        gu, grads = layer.backward(c.gf)
        return [f, gu, *[grads[k] for k in sorted(grads)]]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        held = step()
    for _ in range(3):
        c.u.mul_(0.75)
        c.gf.add_(0.125)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
