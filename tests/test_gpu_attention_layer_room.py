"""The attention layer with room in front of the first and behind the last sub-graph: what those
rows hold, NaN and infinity among it, reaches no result and no gradient."""

import pytest

from tests.helpers import announce
from tests.test_gpu_attention_layer import Setup, env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(bounds=[5, 70, 70, 200, 290]), dict(bounds=[0, 299], hd=40, rot=24, dim=3, cap=0.0, layout=1),
                                dict(bounds=[1, 300], norm=False), dict(bounds=[8, 8], distance=False)])
@pytest.mark.parametrize("eps", [1e-6, 0.0])
def test_rows_of_no_segment(env, kw, dtype, eps):  # noqa: F811
    dm, lib, torch = env
    announce(dtype, kw, eps)
    c = Setup(env, dtype, **kw)
    c.s.eps = eps
    room = torch.ones(c.s.n, dtype=torch.bool, device="cuda")
    room[c.bounds[0]:c.bounds[-1]] = False
    layer = dm.AttentionLayer(lib, c.s)

    def step(u, pos, gf):
        f = layer.forward(c.p, u, pos, c.seg)
        grad_u, grads = layer.backward(gf)
        return {"f": f, "grad_u": grad_u, **grads}

    want = step(c.u, c.pos, c.gf)
    for rows in (float("nan"), float("inf"), 0.0):
        u, pos, gf = (t.clone() for t in (c.u, c.pos, c.gf))
        for t in (u, pos, gf):
            t[room] = rows
        before = [t.clone() for t in (u, pos, gf)]
        got = step(u, pos, gf)
        torch.cuda.synchronize()
        for name, w in want.items():
            assert torch.isfinite(w).all() and torch.equal(got[name], w), (name, rows)
        assert not got["f"][room].any() and not got["grad_u"][room].any()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((u, pos, gf), before))
    if c.bounds[-1] > c.bounds[0]:
        layer2 = Setup(env, dtype, **kw)
        layer2.check()


def test_captured_with_bounds_that_move(env):  # noqa: F811
    """The rows are found from the bounds that a replay has."""
    dm, lib, torch = env
    c = Setup(env, "bf16", n=300, bounds=[3, 100, 250])
    layer = dm.AttentionLayer(lib, c.s)
    c.u[250:], c.gf[250:], c.u[:3] = float("nan"), float("nan"), float("inf")

    def step():
        f = layer.forward(c.p, c.u, c.pos, c.seg)
        gu, grads = layer.backward(c.gf)
        return [f, gu, *[grads[k] for k in sorted(grads)]]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        held = step()
    for bounds in ([3, 100, 250], [10, 30, 120], [3, 3, 249]):
        c.seg.copy_(torch.tensor(bounds, dtype=torch.int32))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.isfinite(w).all() and torch.equal(a, w) for a, w in zip(held, want))


def test_reading_at_points(env):  # noqa: F811
    dm, lib, torch = env
    c = Setup(env, "f32", n=400, bounds=[10, 150, 151, 390])
    qb = torch.tensor([1, 3, 4, 6], dtype=torch.int32, device="cuda")
    u, pos = torch.randn(9, c.s.d, device="cuda"), torch.rand(9, c.s.dim, device="cuda")
    layer = dm.AttentionLayer(lib, c.s)
    want = layer.read(c.p, u, pos, c.u, c.pos, qb, c.seg)
    u[0], u[6:], pos[6:] = float("nan"), float("inf"), float("nan")
    c.u[:10], c.u[390:], c.pos[390:] = float("inf"), float("nan"), float("nan")
    got = layer.read(c.p, u, pos, c.u, c.pos, qb, c.seg)
    assert torch.equal(got, want) and not got[0].any() and not got[6:].any()


def test_refusals(env):  # noqa: F811
    """What would be spread over the rows of no segment is refused: it is no matrix of the layer's."""
    dm, lib, torch = env
    c = Setup(env, "f32", n=64, d=64, bounds=[2, 60])
    layer = dm.AttentionLayer(lib, c.s)
    bad = [(c.u[:, 0], c.pos, c.seg), (c.u, c.pos[:, 0], c.seg), (c.u, c.pos, c.seg.cpu()), (c.u, c.pos, c.seg[:1]),
           (c.u, c.pos, c.seg.long()), (c.u, c.pos, 5), (c.u, c.pos, 1.5)]
    for u, pos, seg in bad:
        with pytest.raises(dm.DsmpError) as e:
            layer.forward(c.p, u, pos, seg)
        assert e.value.status == dm.INVALID_ARG
    layer.forward(c.p, c.u, c.pos, c.seg)
    for g in (c.gf[0], c.gf[:10], c.gf[:, :1]):
        with pytest.raises(dm.DsmpError) as e:
            layer.backward(g)
        assert e.value.status == dm.INVALID_ARG


def test_on_a_stream_of_its_own(env):  # noqa: F811
    """A layer made on one stream and run on another at once: nothing of it waits on the first."""
    dm, lib, torch = env
    c = Setup(env, "f32", n=300, bounds=[5, 100, 250])
    c.u[250:], c.gf[:5] = float("nan"), float("inf")
    layer = dm.AttentionLayer(lib, c.s)
    want = layer.forward(c.p, c.u, c.pos, c.seg), *layer.backward(c.gf)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda")
    for _ in range(20):
        busy = torch.mm(busy, busy).clamp_(-1, 1)
    other = dm.AttentionLayer(lib, c.s)
    with torch.cuda.stream(side):
        got = other.forward(c.p, c.u, c.pos, c.seg), *other.backward(c.gf)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert all(torch.equal(got[2][k], want[2][k]) for k in want[2])
