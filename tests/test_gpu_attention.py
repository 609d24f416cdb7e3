"""GPU parity of attention within packed segments, forward and backward, against the
float64 oracle, element by element within the bounds that it derives."""

import numpy as np
import pytest

from oracle import attention as oa
from tests.helpers import announce, gpu_lib

pytestmark = pytest.mark.gpu

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
# the hardware's power and reciprocal are within 2^-22 of 1 - 2 / (1 + e^2x); float32 scores take the library's tanh
CAP_ABS = {"f32": 2.0 ** -23, "bf16": 2.0 ** -21}


@pytest.fixture(scope="module")
def env():
    return gpu_lib()


def f64(t):
    return t.detach().double().cpu().numpy()


class Case:
    """Inputs of packed segments; rows of no segment hold NaN, outputs start as a mark that has to stay there.
    slices: all matrices are columns of wider ones."""

    def __init__(self, env, q_bounds, k_bounds, H, Hk, hd, dtype, dim=0, cap=0.0, scale=None, seed=0, room=0, slices=False,
                 spread=1.0):
        dm, lib, torch = env
        self.dm, self.lib, self.torch = dm, lib, torch
        self.nq, self.nk = q_bounds[-1] + room, k_bounds[-1] + room
        self.qb, self.kb, self.H, self.Hk, self.hd, self.name = q_bounds, k_bounds, H, Hk, hd, dtype
        self.dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.scale, self.cap, self.dim = hd ** -0.5 if scale is None else scale, cap, dim
        g = np.random.default_rng(seed + 17 * self.nq + self.nk + hd)
        self.slices = slices
        cuda = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731

        def matrix(n, width, bounds):
            w = g.normal(size=(n, width)) * spread
            w[:bounds[0]] = np.nan
            w[bounds[-1]:] = np.nan
            return self.wide(cuda(w).to(self.dt))

        self.q, self.k, self.v = matrix(self.nq, H * hd, q_bounds), matrix(self.nk, Hk * hd, k_bounds), matrix(self.nk, Hk * hd, k_bounds)
        self.do = matrix(self.nq, H * hd, q_bounds)
        self.at = {}
        if dim:
            self.at = dict(pos=cuda(g.random((self.nq, dim))), k_pos=cuda(g.random((self.nk, dim))),
                           slopes=cuda(8.0 * g.random(H)))
        i32 = lambda b: torch.tensor(b, dtype=torch.int32, device="cuda")  # noqa: E731
        self.at.update(segments=i32(q_bounds), k_segments=i32(k_bounds))
        self.desc = dm.attention_desc(H, Hk, hd, {"f32": dm.F32, "bf16": dm.BF16}[dtype], dim=dim, scale=self.scale, cap=cap)

    def wide(self, t):
        if not self.slices:
            return t
        w = self.torch.full((t.shape[0], t.shape[1] + 24), float("nan"), dtype=t.dtype, device=t.device)
        w[:, 16:16 + t.shape[1]] = t
        return w[:, 16:16 + t.shape[1]]

    def marked(self, like):
        return self.wide(self.torch.full_like(like, 77.0))

    def heads(self, t, H):
        return f64(t).reshape(t.shape[0], H, self.hd)

    def places(self):
        return () if not self.dim else (f64(self.at["pos"]), f64(self.at["k_pos"]), f64(self.at["slopes"]))

    def forward(self, **kw):
        out, lse = self.marked(self.q), self.torch.full((self.nq, self.H), 77.0, device="cuda")
        self.lib.dsmp_attention_forward(self.desc, self.q, self.k, self.v, out=out, lse=lse, **self.at, **kw)
        return out, lse

    def backward(self, out, lse, **kw):
        g = [self.marked(t) for t in (self.q, self.k, self.v)]
        self.lib.dsmp_attention_backward(self.desc, self.q, self.k, self.v, out, lse, self.do, grad_q=g[0], grad_k=g[1],
                                         grad_v=g[2], **self.at, **kw)
        return g

    def near(self, what, got, want, tol, bounds):
        inside = slice(bounds[0], bounds[-1])
        assert (got[:bounds[0]] == 77.0).all() and (got[bounds[-1]:] == 77.0).all(), what + ": rows of no segment"
        got, want, tol = got[inside], want[inside], tol[inside]
        assert not np.isnan(got).any(), what
        same = got == want                                        # infinities of rows without keys
        with np.errstate(invalid="ignore"):
            far = np.where(same, 0.0, np.abs(got - want) / np.maximum(tol, 1e-300))
        assert (far <= 1.0).all(), (what, float(far.max()))

    def check(self, backward=True):
        err = oa.Errors(HALF_STEP[self.name], CAP_ABS[self.name])
        q, k, v, do = self.heads(self.q, self.H), self.heads(self.k, self.Hk), self.heads(self.v, self.Hk), self.heads(self.do, self.H)
        args = (self.qb, self.kb, self.scale, self.cap, *(self.places() or (None, None, None)))
        out, lse = self.forward()
        self.torch.cuda.synchronize()
        w_out, w_lse, e_out, e_lse = oa.attention(q, k, v, *args, err=err)
        self.near("lse", f64(lse), w_lse, e_lse, self.qb)
        self.near("out", self.heads(out, self.H), w_out, e_out, self.qb)
        if not backward:
            return
        got = self.backward(out, lse)
        self.torch.cuda.synchronize()
        res = oa.attention_backward(q, k, v, do, *args, err=err)
        for i, (what, H, b) in enumerate((("dq", self.H, self.qb), ("dk", self.Hk, self.kb), ("dv", self.Hk, self.kb))):
            self.near(what, self.heads(got[i], H), res[i], res[3 + i], b)


SIZES = [
    ([0, 1], [0, 1]), ([0, 1], [0, 33]), ([0, 33], [0, 1]), ([0, 31], [0, 65]), ([0, 127], [0, 127]), ([0, 129], [0, 128]),
    ([0, 5, 5, 70], [0, 64, 90, 90]),          # no queries in the second, no keys in the third
    ([3, 40, 41, 160], [2, 34, 162, 163]),     # room in front of the first and behind the last
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", range(len(SIZES)))
def test_lengths_and_segments(env, sizes, dtype):
    qb, kb = SIZES[sizes]
    announce(dtype, qb, kb)
    Case(env, qb, kb, 2, 1, 32, dtype, dim=2, room=5).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [8, 16, 40, 64, 72, 128])
@pytest.mark.parametrize("H,Hk", [(1, 1), (6, 2), (8, 1)])
def test_heads(env, H, Hk, hd, dtype):
    announce(dtype, H, Hk, hd)
    Case(env, [0, 50, 83], [0, 130, 201], H, Hk, hd, dtype, slices=True, room=1).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("dim,cap", [(0, 5.0), (0, 1024.0), (1, 0.0), (1, 2.0), (2, 3.0), (3, 0.0), (3, 20.0)])
def test_scores(env, dim, cap, hd, dtype):
    announce(dtype, dim, cap, hd)
    Case(env, [0, 70], [0, 100], 4, 2, hd, dtype, dim=dim, cap=cap, scale=0.3).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("dim,cap", [(0, 0.0), (0, 5.0), (2, 0.0), (3, 0.0), (3, 5.0)])
def test_large_tiles(env, dim, cap, hd, dtype):
    """Enough tiles of 128 rows to fill the card: many heads of a few short segments, keys shared by none."""
    announce(dtype, dim, cap, hd)
    H = 128
    Case(env, [1, 131, 140, 200], [1, 98, 170, 200], H, H, hd, dtype, dim=dim, cap=cap, room=2).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,qb,kb,dim", [(8, 2, [0, 1], [0, 5000], 3), (4, 4, [2, 3, 3, 8], [0, 4000, 4100, 9001], 0),
                                            (16, 1, [0, 1, 2], [0, 0, 7777], 2)])
def test_few_queries_over_many_keys(env, H, Hk, qb, kb, dim, dtype):
    """Cut over the keys; a split may have no keys of a short segment, a segment none at all."""
    announce(dtype, H, Hk, qb, kb)
    c = Case(env, qb, kb, H, Hk, 64, dtype, dim=dim, room=3)
    assert c.lib.dsmp_attention_workspace(c.desc, c.nq, c.nk, c.at["segments"], c.at["k_segments"])[0] > 0
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nq,nk,H", [(700, 20, 128), (20, 700, 128)])
def test_many_rows_and_few_keys_and_the_other_way(env, nq, nk, H, dtype):
    """Tiles of 128 on one side of the backward pass and of 32 on the other."""
    announce(dtype, nq, nk)
    Case(env, [0, nq], [0, nk], H, H, 16, dtype, dim=1).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_that_rise_from_tile_to_tile(env, dtype):
    """Each later key scores higher: the running maximum is passed by more than its slack again and again, and
    the first keys' weights are below the smallest float32 (88 and more below the sum)."""
    c = Case(env, [0, 40], [0, 1000], 2, 2, 16, dtype, scale=1.0)
    c.k.copy_((c.torch.arange(1000, device="cuda")[:, None] * 0.06).expand(1000, 32))
    g = c.torch.Generator(device="cuda")
    g.manual_seed(11)
    c.q.copy_(c.torch.rand(40, 32, generator=g, device="cuda") * 0.2)
    announce(dtype)
    c.check()
    assert float(c.forward()[1].max()) > 92.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_segments(env, dtype):
    """Segments found from their bounds 64 at a time, over three rounds."""
    g = np.random.default_rng(5)
    qb = np.concatenate([[0], np.cumsum(g.integers(0, 3, 5000))]).tolist()
    kb = np.concatenate([[0], np.cumsum(g.integers(0, 4, 5000))]).tolist()
    announce(dtype, qb[-1], kb[-1])
    Case(env, qb, kb, 1, 1, 16, dtype, dim=1).check()


def test_segments_as_a_count_or_none(env):
    dm, lib, torch = env
    c = Case(env, [0, 60, 120, 180], [0, 60, 120, 180], 2, 2, 32, "bf16")
    out, lse = c.forward()
    o2, l2 = lib.dsmp_attention_forward(c.desc, c.q, c.k, c.v, segments=3)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    one = Case(env, [0, 180], [0, 90], 2, 2, 32, "bf16", dim=1)
    out, lse = one.forward()
    o2, l2 = lib.dsmp_attention_forward(one.desc, one.q, one.k, one.v, pos=one.at["pos"], k_pos=one.at["k_pos"],
                                        slopes=one.at["slopes"])
    assert torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sharp_and_large_scores(env, dtype):
    """Rows that one key takes all of; scores of some hundreds (their bounds grow with them)."""
    c = Case(env, [0, 64], [0, 200], 2, 1, 64, dtype, scale=2.0, spread=2.0)
    announce(dtype)
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [-0.4, 0.0])
@pytest.mark.parametrize("dim,cap", [(0, 0.0), (2, 0.0), (2, 3.0)])
def test_scales_of_any_sign(env, scale, dim, cap, dtype):
    announce(dtype, scale, dim, cap)
    Case(env, [0, 70], [0, 150], 2, 1, 32, dtype, dim=dim, cap=cap, scale=scale).check()


def test_nan_and_infinity_stay_in_their_segment(env):
    dm, lib, torch = env
    c = Case(env, [0, 40, 80], [0, 70, 140], 2, 2, 32, "bf16", dim=2)
    clean = c.forward()
    g_clean = c.backward(*clean)
    c.k[100], c.v[101], c.v[102] = float("nan"), float("inf"), float("nan")
    c.at["k_pos"][105] = float("nan")
    out, lse = c.forward()
    g = c.backward(out, lse)
    torch.cuda.synchronize()
    assert torch.equal(out[:40], clean[0][:40]) and torch.equal(lse[:40], clean[1][:40])
    assert out[40:].isnan().all()
    assert torch.equal(g[0][:40], g_clean[0][:40])
    assert all(torch.equal(g[i][:70], g_clean[i][:70]) for i in (1, 2))
    assert g[0][40:].isnan().all()


def test_no_rows_and_no_keys(env):
    dm, lib, torch = env
    d = dm.attention_desc(2, 2, 32, dm.BF16)
    z, x = torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(7, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = lib.dsmp_attention_forward(d, z, x, x)
    assert out.shape == (0, 64) and lse.shape == (0, 2)
    gq, gk, gv = lib.dsmp_attention_backward(d, z, x, x, out, lse, z)
    assert gq.shape == (0, 64) and not gk.any() and not gv.any()
    out, lse = lib.dsmp_attention_forward(d, x, z, z)
    assert not out.any() and (lse == -float("inf")).all()
    gq, gk, gv = lib.dsmp_attention_backward(d, x, z, z, out, lse, x)
    assert not gq.any() and gk.shape == (0, 64)


@pytest.mark.parametrize("H,n", [(2, 500), (128, 500)])
def test_results_are_the_same_on_every_run_and_scratch_stays_inside(env, H, n):
    dm, lib, torch = env
    c = Case(env, [0, 77, n], [0, 180, n], H, H, 32, "bf16", dim=3, cap=9.0)
    f, b = lib.dsmp_attention_workspace(c.desc, c.nq, c.nk, c.at["segments"], c.at["k_segments"])
    first = None
    for _ in range(3):
        guard = [torch.full((size + 512,), 91, dtype=torch.uint8, device="cuda") for size in (f, b)]
        out, lse = c.forward(ws=guard[0][256:256 + f])
        got = [out, lse, *c.backward(out, lse, ws=guard[1][256:256 + b])]
        torch.cuda.synchronize()
        assert all((w[:256] == 91).all() and (w[-256:] == 91).all() for w in guard)
        first = got if first is None else first
        assert all(torch.equal(x, y) for x, y in zip(got, first))


def test_scratch_of_splits_stays_inside(env):
    dm, lib, torch = env
    c = Case(env, [0, 3], [0, 6000], 4, 2, 40, "bf16")
    f, _ = lib.dsmp_attention_workspace(c.desc, c.nq, c.nk, c.at["segments"], c.at["k_segments"])
    assert f > 0
    w = torch.full((f + 512,), 91, dtype=torch.uint8, device="cuda")
    want = c.forward()
    got = c.forward(ws=w[256:256 + f])
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert (w[:256] == 91).all() and (w[-256:] == 91).all()


@pytest.mark.parametrize("nq,nk", [(300, 300), (2, 4000)])
def test_captured_calls_replay(env, nq, nk):
    """Forward and backward in one graph, replayed on new values between eager calls of larger inputs."""
    dm, lib, torch = env
    c = Case(env, [0, nq], [0, nk], 4, 2, 64, "bf16", dim=2)
    big = Case(env, [0, 2 * nq], [0, 2 * nk], 4, 2, 64, "bf16", dim=2)
    c.backward(*c.forward())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out, lse = lib.dsmp_attention_forward(c.desc, c.q, c.k, c.v, **c.at)
        grads = lib.dsmp_attention_backward(c.desc, c.q, c.k, c.v, out, lse, c.do, **c.at)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for _ in range(4):
        for t in (c.q, c.k, c.v, c.do):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        big.backward(*big.forward())
        graph.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in (out, lse, *grads)]
        o, l = c.forward()
        want = [o, l, *c.backward(o, l)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(kept, want))


def test_two_streams_at_once(env):
    dm, lib, torch = env
    a, b = (Case(env, [0, 200], [0, 6000], 4, 2, 64, "bf16", seed=s) for s in (1, 2))
    want = [[c.forward()[0], *c.backward(*c.forward())] for c in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for _ in range(3):
        for i, c in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                f = c.forward()
                got[i] = [f[0], *c.backward(*f)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for u, v in zip(got, want) for x, y in zip(u, v))


def test_gradients_match_differences_of_the_kernels_own_results(env):
    """float32: the loss at +-h along a direction, against the gradients.  The loss's error is at most the sum
    of |do| times the bounds of out; the difference itself misses third derivatives times h^2 / 6."""
    dm, lib, torch = env
    c = Case(env, [0, 20, 48], [0, 30, 75], 2, 1, 32, "f32", dim=2, cap=4.0)
    out, lse = c.forward()
    grads = c.backward(out, lse)
    err = oa.Errors(HALF_STEP["f32"], CAP_ABS["f32"])
    e_out = oa.attention(c.heads(c.q, 2), c.heads(c.k, 1), c.heads(c.v, 1), c.qb, c.kb, c.scale, c.cap, *c.places(), err=err)[2]
    noise = float((np.abs(c.heads(c.do, 2)) * e_out).sum())
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    for t, grad in zip((c.q, c.k, c.v), grads):
        d = torch.randn(t.shape, generator=g, device="cuda")
        kept, losses = t.clone(), {}
        for h in (2.0 ** -6, 2.0 ** -7):
            for sign in (1, -1):
                t.copy_(kept + sign * h * d)
                losses[sign * h] = float((c.forward()[0].double() * c.do.double()).sum())
        t.copy_(kept)
        # two steps: Richardson's combination is free of the third derivative
        d1, d2 = ((losses[h] - losses[-h]) / (2 * h) for h in (2.0 ** -6, 2.0 ** -7))
        diff = (4 * d2 - d1) / 3
        want = float((grad.double() * d.double()).sum())
        assert abs(diff - want) <= 2 * noise * 2 ** 7 * (4 / 3 + 1 / 6) + abs(d2 - d1), (diff, want)


def test_refusals(env):
    dm, lib, torch = env
    c = Case(env, [0, 8], [0, 8], 2, 1, 32, "bf16", dim=2)

    def refused(status, desc=c.desc, q=c.q, k=c.k, v=c.v, **kw):
        with pytest.raises(dm.DsmpError) as e:
            lib.dsmp_attention_forward(desc, q, k, v, **{**c.at, **kw})
        assert e.value.status == status, e.value

    bad = dm.INVALID_ARG
    refused(bad, q=c.q.float())
    refused(bad, q=c.q[:, :32])
    refused(bad, k=c.k[:4])
    refused(bad, q=c.q.cpu())
    refused(bad, pos=None)
    refused(bad, slopes=c.at["slopes"][:1])
    refused(bad, slopes=None)
    refused(bad, k_segments=torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda"))
    refused(bad, segments=torch.tensor([0, 8], device="cuda"))
    refused(bad, ws=torch.empty(4, device="cuda"))
    odd = torch.zeros(8, 72, dtype=torch.bfloat16, device="cuda")
    refused(bad, q=odd[:, 4:68])                                    # rows that are not 16-byte aligned
    refused(bad, q=torch.zeros(8, 68, dtype=torch.bfloat16, device="cuda")[:, :64])
    refused(dm.UNSUPPORTED, desc=dm.attention_desc(2, 1, 12, dm.BF16, dim=2), q=c.q[:, :24], k=c.k[:, :12], v=c.v[:, :12])
    out, lse = c.forward()
    with pytest.raises(dm.DsmpError) as e:
        lib.dsmp_attention_backward(c.desc, c.q, c.k, c.v, out, lse[:4], c.do, **c.at)
    assert e.value.status == bad
    with pytest.raises(dm.DsmpError) as e:
        lib.dsmp_attention_backward(c.desc, c.q, c.k, c.v, out, lse, c.do, ws=torch.empty(8, dtype=torch.uint8, device="cuda"), **c.at)
    assert e.value.status == dm.WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_tiles_of_many_segments(env, dtype):
    """More segments than are ordered by their length, in tiles of 128 rows."""
    g = np.random.default_rng(8)
    qb, kb = (np.concatenate([[0], np.cumsum(g.integers(90, 200, 70))]).tolist() for _ in range(2))
    announce(dtype, qb[-1], kb[-1])
    Case(env, qb, kb, 16, 16, 32, dtype, dim=3).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk", [(256, 1), (255, 51)])
def test_most_heads(env, H, Hk, dtype):
    """More rows to a query than a tile has, and heads whose number is no power of two."""
    announce(dtype, H, Hk)
    Case(env, [0, 3, 10], [0, 90, 151], H, Hk, 16, dtype, dim=2).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,n", [(1, 200), (128, 200)])
def test_wrong_bounds_leave_other_memory_alone(env, H, n, dtype):
    """Bounds that descend, are negative or past the end: the kernels hold them to the arrays."""
    dm, lib, torch = env
    c = Case(env, [0, n], [0, n], H, H, 32, dtype, dim=2)
    bounds = torch.tensor([-7, 60, 20, 99999, 2 ** 31 - 1, -(2 ** 31), 150], dtype=torch.int32, device="cuda")
    at = {**c.at, "segments": bounds, "k_segments": bounds.flip(0).contiguous()}
    announce(dtype, H)
    outs = [torch.full((3 * n, 32 * H), 7.0, dtype=c.q.dtype, device="cuda") for _ in range(4)]
    lse = torch.full((3 * n, H), 7.0, device="cuda")
    mid = slice(n, 2 * n)
    lib.dsmp_attention_forward(c.desc, c.q, c.k, c.v, out=outs[0][mid], lse=lse[mid], **at)
    lib.dsmp_attention_backward(c.desc, c.q, c.k, c.v, outs[0][mid], lse[mid], c.do, grad_q=outs[1][mid], grad_k=outs[2][mid],
                                grad_v=outs[3][mid], **at)
    torch.cuda.synchronize()
    for t in (*outs, lse):
        assert (t[:n] == 7).all() and (t[2 * n:] == 7).all()


def test_captured_call_takes_the_bounds_of_its_replay(env):
    dm, lib, torch = env
    a, b = (Case(env, [0, x, 90], [0, y, 150], 2, 1, 32, "bf16", dim=2, seed=4) for x, y in ((30, 100), (71, 9)))
    a.backward(*a.forward())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        out, lse = lib.dsmp_attention_forward(a.desc, a.q, a.k, a.v, **a.at)
        grads = lib.dsmp_attention_backward(a.desc, a.q, a.k, a.v, out, lse, a.do, **a.at)
    for name in ("segments", "k_segments"):
        a.at[name].copy_(b.at[name])
    for _ in range(3):
        graph.replay()
        o, l = a.forward()
        want = [o, l, *a.backward(o, l)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((out, lse, *grads), want))


@pytest.mark.parametrize("nq,nk", [(50, 90), (3, 2000)])
def test_weights_of_small_calls_keep_sixteen_bits(env, nq, nk):
    """bfloat16: P is a sum of two values, within 2^-16 of it (what is left after the first rounding, 2^-8, is rounded
    to 2^-8 of that).  A score is exact products added in float32, 34 roundings of 2^-24 of sum |q k| scale < 16: below
    2^-14.9 of P; power, sum and logarithm stay below 2^-20.  So out and dv are within 2^-14 sum P |v| and half a step of
    their own, 2^-8."""
    c = Case(env, [0, nq], [0, nk], 4, 2, 32, "bf16")
    announce(nq, nk)
    out, lse = c.forward()
    _, _, dv = c.backward(out, lse)
    q, k, v, do = (c.heads(t, h) for t, h in ((c.q, 4), (c.k, 2), (c.v, 2), (c.do, 4)))
    want_dv, room = np.zeros_like(v), np.zeros_like(v)
    for a in range(4):
        z = c.scale * q[:, a] @ k[:, a // 2].T
        assert (c.scale * np.abs(q[:, a]) @ np.abs(k[:, a // 2]).T).max() < 16
        P = np.exp(z - z.max(1, keepdims=True))
        P /= P.sum(1, keepdims=True)
        o = P @ v[:, a // 2]
        near = 2.0 ** -14 * (P @ np.abs(v[:, a // 2]))
        assert (np.abs(c.heads(out, 4)[:, a] - o) <= 2.0 ** -8 * (np.abs(o) + near) + near).all()
        want_dv[:, a // 2] += P.T @ do[:, a]
        room[:, a // 2] += 2.0 ** -14 * (P.T @ np.abs(do[:, a]))
    assert (np.abs(c.heads(dv, 2) - want_dv) <= 2.0 ** -8 * (np.abs(want_dv) + room) + room).all()


def test_gradients_of_one_key_are_zero(env):
    """bfloat16: the one weight does not depend on the score.  D comes from the weight then: dS = P (e - P e) with
    e = dP - D of the rounded out, |e| <= 2^-7 A, A = sum |dO v|, and P within 2^-14 of 1 (|z| < 32: 34 roundings of 2^-24 of
    it): below 2^-21 A; the sums of dP and D are within 34 2^-24 A of each other in e and cancel but for P's part;
    their rounding, 2^-24 |e|, is less.  So dS is below 2^-20 A; from the rounded out alone it would be about 2^-12 A."""
    n = 40
    c = Case(env, list(range(0, 3 * n + 1, 3)), list(range(n + 1)), 4, 2, 32, "bf16", dim=2)
    announce(n)
    out, lse = c.forward()
    assert float(lse.abs().max()) < 32
    dq, dk, _ = c.backward(out, lse)
    q, k, v, do = (c.heads(t, h) for t, h in ((c.q, 4), (c.k, 2), (c.v, 2), (c.do, 4)))
    room = np.zeros_like(k)
    for a in range(4):
        key = np.arange(3 * n) // 3
        A = c.scale * 2.0 ** -20 * (np.abs(do[:, a]) * np.abs(v[key, a // 2])).sum(1, keepdims=True)
        assert (np.abs(c.heads(dq, 4)[:, a]) <= A * np.abs(k[key, a // 2])).all()
        np.add.at(room[:, a // 2], key, A * np.abs(q[:, a]))
    assert (np.abs(c.heads(dk, 2)) <= room).all()
