"""GPU parity of the pre-norm stack with 8-bit activation checkpoints against
the float64 oracle's norms and layers, composed the same way.

The backward reference takes the kept values and statistics from the stack
itself (what a checkpoint loses is part of the method), so the bar is the
layers' own: 1e-4 (float32), or 2e-2 for each of the layers (bf16 operands).
The kernel networks' inner gradients (W1, b1, W2, b2) jump with decisions near
a kink and are covered by the layer's tests."""

import numpy as np
import pytest

import oracle
from oracle import nnconv as onn
from oracle import norm as on
from tests.helpers import TOL, announce, gpu_lib, rel_err
from workloads import layer_params

pytestmark = pytest.mark.gpu

LAYERS = 3


@pytest.fixture(scope="module")
def env():
    return gpu_lib()


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Setup:
    def __init__(self, env, n, d, h, dtype, segments, checkpoints, seed=0):
        dm, lib, torch = env
        g = np.random.default_rng(seed + n)
        self.pos = g.uniform(0, 1, (n, 2)).astype(np.float32)
        r = float(np.sqrt(12.0 / (np.pi * n)))
        attr = np.concatenate([self.pos, g.normal(size=(n, 1)).astype(np.float32)], 1)
        self.P = [layer_params(g, d, 6, h, h, dtype) for _ in range(LAYERS)]
        self.x = (g.normal(size=(n, d)) + 0.5 * g.normal(size=d)).astype(np.float32)
        self.gamma = [(1 + 0.2 * g.normal(size=d)).astype(np.float32) for _ in range(LAYERS + 1)]
        self.beta = [(0.2 * g.normal(size=d)).astype(np.float32) for _ in range(LAYERS + 1)]
        self.gy = g.normal(size=(n, d)).astype(np.float32)
        self.segments, self.groups, self.dtype = segments, d // 8, dtype
        rp, col = oracle.radius_graph.radius_graph(self.pos, n, r)[:2]
        self.rp, self.col = rp, col
        self.xe = onn.edge_attr(attr, rp, col, "concat")
        cu = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
        graph = lib.dsmp_radius_graph_build(cu(self.pos), n, r)
        assert graph.n_edges == len(col)
        code = dm.BF16 if dtype == "bf16" else dm.F32
        shapes = dm.StackShapes(n, 2, d, h, h, code, LAYERS, self.groups)
        seg = cu(np.array(segments, np.int32)) if isinstance(segments, list) else segments
        self.stack = dm.CheckpointedStack(lib, graph, shapes, segments=seg, checkpoints=checkpoints)
        packed = [lib.dsmp_nnconv_pack(self.stack.conv, {k: cu(v) for k, v in p.items()}) for p in self.P]
        self.args = (packed, [(cu(a), cu(b)) for a, b in zip(self.gamma, self.beta)], cu(attr), cu(self.x))
        self.gyc = cu(self.gy)

    def act(self, l):
        return on.IDENTITY if l == LAYERS else on.SILU

    def conv(self, l, u):
        return onn.forward(self.P[l], self.xe, u, self.rp, self.col, len(u), residual=False)[0]

    def reference(self):
        """y, and every s_l"""
        s, out = self.x.astype(np.float64), []
        for l in range(LAYERS + 1):
            out.append(s)
            u, _ = on.forward(s, self.segments, self.groups, self.gamma[l].astype(np.float64), self.beta[l], self.act(l),
                              1e-5)
            if l < LAYERS:
                s = s + self.conv(l, u)
        return u, out

    def reference_grads(self, streams, stats, exact_last_u):
        """(grad_x, layer gradients, norm gradients) from values t_l of the stream and statistics."""
        conv, norm = [None] * LAYERS, [None] * (LAYERS + 1)
        G, a, b = on.backward(streams[LAYERS], stats[LAYERS], self.segments, self.gamma[LAYERS], self.beta[LAYERS],
                              on.IDENTITY, self.gy)
        norm[LAYERS] = (a, b)
        for l in reversed(range(LAYERS)):
            u = on.act(on.normalised(streams[l], stats[l], self.segments) * self.gamma[l] + self.beta[l], on.SILU)
            if l == LAYERS - 1:
                u = exact_last_u
            conv[l] = onn.backward(self.P[l], self.xe, u, self.rp, self.col, len(u), G, residual=False)
            dx, a, b = on.backward(streams[l], stats[l], self.segments, self.gamma[l], self.beta[l], on.SILU,
                                   conv[l]["grad_h"])
            norm[l] = (a, b)
            G = G + dx
        return G, conv, norm


CASES = [(400, 32, 64, "f32", None), (400, 32, 64, "f32", [0, 150, 150, 400]), (300, 64, 128, "bf16", None),
         (300, 32, 64, "f32", 300)]


@pytest.mark.parametrize("checkpoints", [True, False])
@pytest.mark.parametrize("n,d,h,dtype,segments", CASES)
def test_stack_forward_and_backward(env, n, d, h, dtype, segments, checkpoints):
    announce("stack", n, d, dtype, segments, checkpoints)
    c = Setup(env, n, d, h, dtype, segments, checkpoints)
    st = c.stack
    bar = TOL["f32"] if dtype == "f32" else LAYERS * TOL["bf16"]
    y = st.forward(*c.args)
    want, streams = c.reference()
    assert rel_err(_np(y), want) <= bar
    assert np.array_equal(_np(c.args[3]), c.x.astype(np.float64))      # x is left as it is
    stats = [_np(t) for t in st.stats]
    if checkpoints:
        t = [on.values(k.q.cpu().numpy(), k.scale.cpu().numpy()).astype(np.float64) for k in st.kept]
        for a, b in zip(t, streams):
            # half a step of a block's largest value, and what the forward pass is off
            assert np.abs(a - b).max() <= (0.5 / 127 + bar) * 1.01 * np.abs(b).max()
    else:
        t = [c.x.astype(np.float64)] + [_np(v) for v in st.stream]
    last_u = _np(st._at(st.u, LAYERS - 1))
    gx, conv, norm = st.backward(c.gyc)
    rgx, rconv, rnorm = c.reference_grads(t, stats, last_u)
    assert rel_err(_np(gx), rgx) <= bar, "grad_x"
    for l in range(LAYERS):
        for k in ("dW3", "db3", "dWr", "dbr"):
            assert rel_err(_np(conv[l][k]), rconv[l][k]) <= bar, (l, k)
    for l in range(LAYERS + 1):
        assert rel_err(_np(norm[l]["dgamma"]), rnorm[l][0]) <= bar, (l, "dgamma")
        assert rel_err(_np(norm[l]["dbeta"]), rnorm[l][1]) <= bar, (l, "dbeta")


def test_checkpoints_keep_less_and_change_the_gradients_little(env):
    """A step of a block of 64 normal values is about 2.7 / 127 of their deviation, its
    rounding 0.6 % rms; three layers of it stay within 5 % of the gradients' norm."""
    announce("stack checkpoints")
    a, b = (Setup(env, 2000, 64, 128, "bf16", None, ck) for ck in (True, False))
    ya, yb = a.stack.forward(*a.args), b.stack.forward(*b.args)
    assert np.array_equal(_np(ya), _np(yb))                            # the forward pass does not change
    assert a.stack.kept_bytes() < 0.4 * b.stack.kept_bytes()
    (ga, ca, na), (gb, cb, nb) = a.stack.backward(a.gyc), b.stack.backward(b.gyc)

    def far(u, v):
        return float((u.double() - v.double()).norm() / v.double().norm())

    assert far(ga, gb) <= 0.05
    for l in range(LAYERS):
        for k in cb[l]:
            assert far(ca[l][k], cb[l][k]) <= 0.05, (l, k)
    for l in range(LAYERS + 1):
        for k in nb[l]:
            assert far(na[l][k], nb[l][k]) <= 0.05, (l, k)


def test_two_steps_give_the_same_bits(env):
    announce("stack determinism")
    c = Setup(env, 500, 32, 64, "f32", [0, 100, 500], True)
    runs = []
    for _ in range(2):
        y = c.stack.forward(*c.args).clone()
        gx, conv, norm = c.stack.backward(c.gyc)
        runs.append([y, gx.clone()] + [v for m in conv + norm for v in m.values()])
    for u, v in zip(*runs):
        assert np.array_equal(_np(u), _np(v))


def test_refuses_graphs_with_halo_rows(env):
    dm, lib, torch = env
    announce("stack refusals")
    g = lib.dsmp_radius_graph_build(torch.rand(50, 2, device="cuda"), 40, 0.3)
    for shapes in (dm.StackShapes(40, 2, 32, 64, 64, dm.F32, 2, 4), dm.StackShapes(50, 2, 32, 64, 64, dm.F32, 0, 4)):
        with pytest.raises(dm.DsmpError) as e:
            dm.CheckpointedStack(lib, g, shapes)
        assert e.value.status == dm.INVALID_ARG


@pytest.mark.parametrize("checkpoints", [True, False])
@pytest.mark.parametrize("n,d,h,dtype,segments", [CASES[1], CASES[2]])
def test_backward_again_with_another_gradient(env, n, d, h, dtype, segments, checkpoints):
    """A second and a third backward of one forward pass: the gradients of the new grad_y, and the
    same bits where it is the same."""
    dm, lib, torch = env
    announce("stack backward again", n, d, dtype, segments, checkpoints)
    c = Setup(env, n, d, h, dtype, segments, checkpoints)
    st = c.stack
    bar = TOL["f32"] if dtype == "f32" else LAYERS * TOL["bf16"]
    st.forward(*c.args)
    stats = [_np(t) for t in st.stats]
    last_u = st._at(st.u, LAYERS - 1).clone()
    if checkpoints:
        t = [on.values(k.q.cpu().numpy(), k.scale.cpu().numpy()).astype(np.float64) for k in st.kept]
        last_u = lib.dsmp_group_norm_restore(st.norm, st.kept[LAYERS - 1], st.stats[LAYERS - 1], *c.args[1][LAYERS - 1],
                                             segments=st.segments)
    else:
        t = [c.x.astype(np.float64)] + [_np(v) for v in st.stream]
    st.backward(c.gyc)
    c.gy = np.random.default_rng(99).normal(size=c.gy.shape).astype(np.float32)
    gyc = torch.from_numpy(c.gy).cuda()
    runs = []
    for _ in range(2):
        gx, conv, norm = st.backward(gyc)
        runs.append([gx.clone()] + [v.clone() for m in conv + norm for v in m.values()])
    for u, v in zip(*runs):
        assert np.array_equal(_np(u), _np(v))
    rgx, rconv, rnorm = c.reference_grads(t, stats, _np(last_u))
    assert rel_err(_np(gx), rgx) <= bar, "grad_x"
    for l in range(LAYERS):
        for k in ("dW3", "db3", "dWr", "dbr"):
            assert rel_err(_np(conv[l][k]), rconv[l][k]) <= bar, (l, k)
    for l in range(LAYERS + 1):
        assert rel_err(_np(norm[l]["dgamma"]), rnorm[l][0]) <= bar, (l, "dgamma")
        assert rel_err(_np(norm[l]["dbeta"]), rnorm[l][1]) <= bar, (l, "dbeta")
