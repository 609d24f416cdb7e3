"""GPU parity of the group norm (forward, restored, backward) and of the 8-bit
checkpoints against the float64 oracle.

Checkpoints are compared bit for bit.  Floating outputs are held element by
element to bounds that follow from the operations, with u = 2^-24:
  xn   16 u (max|t| rstd + |xn|): the joined means and squares, a difference, a product
  z    |gamma| that, + 4 u (|z| + |beta|)
  y    1.13 (the largest slope of any activation) times that, + 8 u (1 + |z|) + 3e-7 |z|
       for the exponentials and the published polynomial of the normal tail
  w    |dy| (0.8 (the largest second derivative) the bound of z + 1e-6)
  A, B the mean of the bounds of their terms, + 32 u times the mean magnitude
  outputs in bfloat16 add 2^-8 |value| (half a unit in the last place), with 1 % to spare
"""

import math

import numpy as np
import pytest

from oracle import norm as on
from tests.helpers import announce, gpu_lib

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = 2.0 ** -8 * 1.01


@pytest.fixture(scope="module")
def env():
    return gpu_lib()


def _np(t):
    return t.detach().float().cpu().numpy()


def bits(t):
    """Bytes of a tensor's values (NaN included in comparisons)."""
    import torch
    return t.contiguous().view(torch.uint8).cpu()


class Case:
    """Inputs on the GPU and as float64, with a slope's kink kept away from."""

    def __init__(self, torch, n, C, G, segments=None, x="f32", y="f32", act=on.SILU, eps=1e-5, seed=0, offset=1.0,
                 affine=True, addend=False):
        g = np.random.default_rng(seed + 7 * n + C)
        self.torch, self.n, self.C, self.G, self.act, self.eps = torch, n, C, G, act, eps
        self.dt = {"f32": torch.float32, "bf16": torch.bfloat16}
        self.x_name, self.y_name = x, y
        self.segments = segments
        xv = g.normal(size=(n, C)) * np.exp(0.3 * g.normal(size=C)) + offset * g.normal(size=C)
        self.x = torch.tensor(xv, dtype=torch.float32, device="cuda").to(self.dt[x])
        self.addend = None
        t = self.x
        if addend:
            self.addend = torch.tensor(g.normal(size=(n, C)), dtype=torch.float32, device="cuda").to(self.dt[x])
            t = (self.x.float() + self.addend.float()).to(self.dt[x])
        self.t = t
        f = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
        self.gamma = f(1 + 0.3 * g.normal(size=C)) if affine else None
        self.beta = f(0.3 * g.normal(size=C)) if affine else None
        self.ga64 = _np(self.gamma).astype(np.float64) if affine else np.ones(C)
        self.be64 = _np(self.beta).astype(np.float64) if affine else np.zeros(C)
        self.t64 = _np(t).astype(np.float64)
        self.dy = f(g.normal(size=(n, C)))
        self.grad_addend = f(g.normal(size=(n, C)))

    def desc(self, dm):
        code = {"f32": dm.F32, "bf16": dm.BF16}
        return dm.norm_desc(self.C, self.G, code[self.x_name], code[self.y_name], self.act, self.eps)

    def seg(self):
        return (self.torch.tensor(self.segments, dtype=self.torch.int32, device="cuda")
                if isinstance(self.segments, list) else self.segments)

    def away_from_kink(self, z):
        """ReLU's slope has a jump at zero: no gradient enters within 1e-3 of it."""
        if self.act == on.RELU:
            self.dy[self.torch.tensor(np.abs(z) < 1e-3, device="cuda")] = 0.0

    def bounds(self, t64, stats):
        """(xn, z, and their error bounds) of rows t64."""
        xn = on.normalised(t64, stats, self.segments)
        z = xn * self.ga64 + self.be64
        b = on.bounds(self.n, self.segments)
        row = np.repeat(np.arange(len(b) - 1), np.diff(b))
        rstd = np.repeat(stats[row, :, 1], self.C // self.G, 1)
        big = np.abs(t64).max() if t64.size else 0.0
        exn = 16 * U * (big * rstd + np.abs(xn))
        ez = np.abs(self.ga64) * exn + 4 * U * (np.abs(z) + np.abs(self.be64))
        return xn, z, exn, ez, rstd, row

    def check_y(self, y, t64, stats, what="y"):
        xn, z, exn, ez, _, _ = self.bounds(t64, stats)
        ref = on.act(z, self.act)
        tol = 1.13 * ez + 8 * U * (1 + np.abs(z)) + 3e-7 * np.abs(z)
        tol = tol + (BF * (np.abs(ref) + tol) if self.y_name == "bf16" else U * np.abs(ref))
        err = np.abs(_np(y).astype(np.float64) - ref)
        assert (err <= tol).all(), (what, float((err / tol).max()))

    def check_stats(self, got, t64):
        ref = on.statistics(t64, self.segments, self.G, self.eps)
        got = _np(got).astype(np.float64)
        big = np.abs(t64).max() if t64.size else 0.0
        assert (np.abs(got[:, :, 0] - ref[:, :, 0]) <= 16 * U * big).all()
        # the squares lose what the means do: twice 16 u max|t| sigma
        assert (np.abs(got[:, :, 1] - ref[:, :, 1]) <= ref[:, :, 1] * (32 * U + 32 * U * big * ref[:, :, 1])).all()
        return ref

    def check_backward(self, dx, grads, t64, stats, grad_addend=None, times=1):
        xn, z, exn, ez, rstd, row = self.bounds(t64, stats)
        dy = _np(self.dy).astype(np.float64)
        ref, dgamma, dbeta = on.backward(t64, stats, self.segments, self.ga64, self.be64, self.act, dy)
        w = dy * on.act_slope(z, self.act)
        ew = np.abs(dy) * (0.8 * ez + 1e-6) + 4 * U * np.abs(w)
        ga = np.abs(self.ga64)
        c, nseg = self.C // self.G, len(stats)

        def group_mean(v):
            s = np.zeros((nseg, self.G))
            np.add.at(s, row, v.reshape(self.n, self.G, c).sum(2))
            m = np.bincount(row, minlength=nseg)[:, None] * c
            return np.repeat((s / np.maximum(m, 1))[row], c, 1)

        A, B = group_mean(w * self.ga64), group_mean(w * self.ga64 * xn)
        eA = group_mean(ga * ew) + 32 * U * group_mean(ga * np.abs(w))
        eB = group_mean(ga * (ew * np.abs(xn) + np.abs(w) * exn)) + 32 * U * group_mean(ga * np.abs(w * xn))
        tol = rstd * (ga * ew + eA + np.abs(xn) * eB + exn * np.abs(B)
                      + 8 * U * (ga * np.abs(w) + np.abs(A) + np.abs(xn * B)))
        tol = tol + 16 * U * np.abs(ref)
        if grad_addend is not None:
            ref = ref + _np(grad_addend).astype(np.float64)
            tol = tol + 2 * U * np.abs(ref)
        err = np.abs(_np(dx).astype(np.float64) - ref)
        assert (err <= tol + 1e-30).all(), ("dx", float((err / (tol + 1e-30)).max()))
        if self.gamma is not None:
            tg = (ew * np.abs(xn) + np.abs(w) * exn).sum(0) + 32 * U * np.abs(w * xn).sum(0)
            tb = ew.sum(0) + 32 * U * np.abs(w).sum(0)
            assert (np.abs(_np(grads["dgamma"]) - times * dgamma) <= times * tg + 1e-30).all(), "dgamma"
            assert (np.abs(_np(grads["dbeta"]) - times * dbeta) <= times * tb + 1e-30).all(), "dbeta"


RAGGED = [0, 0, 1, 1, 71, 400, 400, 699, 700, 700]
SHAPES = [
    # n, C, G, segments
    (1, 32, 4, None), (1, 8, 1, [0, 1]), (2, 16, 2, None), (1000, 32, 8, None), (777, 33, 3, None), (2049, 96, 12, None),
    (500, 64, 64, None), (300, 512, 2, None), (130, 257, 1, None), (3, 1, 1, None), (640, 7, 7, None),
    (700, 64, 8, RAGGED), (700, 20, 2, RAGGED), (700, 128, 1, RAGGED), (60, 48, 6, [0, 60, 60, 60]),
    (1000, 64, 16, 8), (4, 200, 25, 2), (9000, 64, 4, None),
    # each row a segment
    (513, 64, 1, 513), (100, 96, 1, 100), (100, 96, 12, 100), (77, 40, 4, 77), (50, 24, 8, 50), (33, 5, 1, 33),
    (1, 3, 1, 1), (65, 512, 2, 65), (1000, 128, 16, 1000), (40, 320, 5, 40), (30, 257, 1, 30), (20, 100, 4, 20),
]


@pytest.mark.parametrize("n,C,G,segments", SHAPES)
def test_forward_restore_backward(env, n, C, G, segments):
    dm, lib, torch = env
    kinds = [on.SILU, on.GELU, on.RELU, on.IDENTITY]
    for i, (x, y) in enumerate([("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")]):
        announce("norm", n, C, G, segments, x, y, kinds[i])
        c = Case(torch, n, C, G, segments, x, y, kinds[i], addend=i % 2 == 1, seed=i)
        d, seg = c.desc(dm), c.seg()
        total = torch.empty_like(c.x) if c.addend is not None else None
        ck = dm.Checkpoint.empty(n, C, c.x.device)
        out, st = lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg, addend=c.addend, sum_out=total,
                                              checkpoint=ck)
        ref = c.check_stats(st, c.t64)
        if total is not None:
            assert torch.equal(total, c.t)
        c.check_y(out, c.t64, ref)
        q, scale = on.checkpoint(_np(c.t))
        assert np.array_equal(ck.q.cpu().numpy(), q) and np.array_equal(ck.scale.cpu().numpy(), scale)
        # without a checkpoint: the same bits
        again, st2 = lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg, addend=c.addend, sum_out=total)
        assert torch.equal(again, out) and torch.equal(st, st2)
        kept = on.values(q, scale).astype(np.float64)
        st64 = _np(st).astype(np.float64)      # the calls below take the statistics as they are
        c.check_y(lib.dsmp_group_norm_restore(d, ck, st, c.gamma, c.beta, segments=seg), kept, st64, "restored")
        for source, t64, ga in ((c.t, c.t64, None), (ck, kept, c.grad_addend)):
            c.away_from_kink(c.bounds(t64, st64)[1])
            dx, grads = lib.dsmp_group_norm_backward(d, source, st, c.gamma, c.beta, c.dy, segments=seg, grad_addend=ga)
            c.check_backward(dx, grads, t64, st64, ga)


def test_without_affine_parameters(env):
    dm, lib, torch = env
    for segments in (None, [0, 100, 300], 300):
        announce("norm no affine", segments)
        c = Case(torch, 300, 48, 6, segments, affine=False)
        d, seg = c.desc(dm), c.seg()
        y, st = lib.dsmp_group_norm_forward(d, c.x, None, None, segments=seg)
        c.check_y(y, c.t64, c.check_stats(st, c.t64))
        dx, grads = lib.dsmp_group_norm_backward(d, c.x, st, None, None, c.dy, segments=seg)
        assert grads == {}
        c.check_backward(dx, None, c.t64, _np(st).astype(np.float64))


@pytest.mark.parametrize("offset", [1e3, 1e5])
def test_large_mean_keeps_its_digits(env, offset):
    """The variance of values far from zero: squares about the mean, not about zero."""
    dm, lib, torch = env
    announce("norm offset", offset)
    for segments in (None, 5000):
        c = Case(torch, 5000, 32, 2, segments)
        c.x = c.x + offset
        c.t64 = _np(c.x).astype(np.float64)
        _, st = lib.dsmp_group_norm_forward(c.desc(dm), c.x, c.gamma, c.beta, segments=c.seg())
        c.check_stats(st, c.t64)


def test_far_out_value_does_not_disturb_the_variance_of_the_rest(env):
    """A value of 1e6 in one group: the other groups keep theirs, its own keeps float32 accuracy."""
    dm, lib, torch = env
    announce("norm outlier")
    c = Case(torch, 4096, 64, 8, None)
    c.x[0, 3] = 1e6
    t64 = _np(c.x).astype(np.float64)
    _, st = lib.dsmp_group_norm_forward(c.desc(dm), c.x, c.gamma, c.beta)
    ref = on.statistics(t64, None, 8, c.eps)
    got = _np(st).astype(np.float64)
    np.testing.assert_allclose(got[0, :, 1], ref[0, :, 1], rtol=64 * U)
    np.testing.assert_allclose(got[0, 1:, 0], ref[0, 1:, 0], atol=64 * U * 10)


@pytest.mark.parametrize("segments", [None, [0, 150, 400], 400])
@pytest.mark.parametrize("C,G", [(64, 8), (33, 3)])
def test_strided_and_unaligned_rows(env, segments, C, G):
    """Column slices of wider matrices at odd places: the same values, and nothing written beside them."""
    dm, lib, torch = env
    n = 400
    for x, y in (("f32", "bf16"), ("bf16", "f32")):
        announce("norm strided", segments, C, x, y)
        c = Case(torch, n, C, G, segments, x, y, addend=True)
        d, seg = c.desc(dm), c.seg()

        def wide(v, at, extra, dtype):
            m = torch.full((n, C + extra), 77.0, dtype=dtype, device="cuda")
            s = m[:, at:at + C]
            if v is not None:
                s.copy_(v)
            return m, s

        def beside(m, at):
            assert (m[:, :at] == 77).all() and (m[:, at + C:] == 77).all()

        _, xs = wide(c.x, 3, 8, c.x.dtype)
        _, ads = wide(c.addend, 1, 2, c.x.dtype)
        sm, ss = wide(None, 5, 9, c.x.dtype)
        ym, ys = wide(None, 1, 5, c.dt[y])
        ck, ck2 = dm.Checkpoint.empty(n, C, "cuda"), dm.Checkpoint.empty(n, C, "cuda")
        want, st0 = lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg, addend=c.addend,
                                                sum_out=torch.empty_like(c.x), checkpoint=ck2)
        _, st = lib.dsmp_group_norm_forward(d, xs, c.gamma, c.beta, segments=seg, addend=ads, sum_out=ss, y=ys,
                                            checkpoint=ck)
        beside(sm, 5)
        beside(ym, 1)
        assert torch.equal(ss, c.t) and torch.equal(ck.q, ck2.q) and torch.equal(ck.scale, ck2.scale)
        c.check_y(ys, c.t64, c.check_stats(st, c.t64))
        rm, rs = wide(None, 2, 6, c.dt[y])
        lib.dsmp_group_norm_restore(d, ck, st, c.gamma, c.beta, segments=seg, y=rs)
        beside(rm, 2)
        c.check_y(rs, on.values(ck.q.cpu().numpy(), ck.scale.cpu().numpy()).astype(np.float64),
                  _np(st).astype(np.float64), "restored")
        _, dys = wide(c.dy, 3, 4, torch.float32)
        _, gas = wide(c.grad_addend, 1, 1, torch.float32)
        dm_, dxs = wide(None, 2, 3, torch.float32)
        _, grads = lib.dsmp_group_norm_backward(d, ss, st, c.gamma, c.beta, dys, segments=seg, grad_addend=gas,
                                                grad_x=dxs)
        beside(dm_, 2)
        c.check_backward(dxs, grads, c.t64, _np(st).astype(np.float64), c.grad_addend)
        lm, ls = wide(None, 1, 2, torch.float32)
        lib.dsmp_checkpoint_load(lib.dsmp_checkpoint_store(xs), ls)
        beside(lm, 1)
        assert np.array_equal(_np(ls), on.values(*on.checkpoint(_np(c.x))))


def test_sum_and_gradient_in_place(env):
    dm, lib, torch = env
    for segments in (None, [0, 10, 500], 500):
        for target in ("x", "addend"):
            announce("norm in place", segments, target)
            c = Case(torch, 500, 64, 8, segments, "bf16", "bf16", addend=True)
            d, seg = c.desc(dm), c.seg()
            x, ad = c.x.clone(), c.addend.clone()
            s = x if target == "x" else ad
            y, st = lib.dsmp_group_norm_forward(d, x, c.gamma, c.beta, segments=seg, addend=ad, sum_out=s)
            assert torch.equal(s, c.t)
            c.check_y(y, c.t64, c.check_stats(st, c.t64))
            g = c.grad_addend.clone()
            _, grads = lib.dsmp_group_norm_backward(d, s, st, c.gamma, c.beta, c.dy, segments=seg, grad_addend=g,
                                                    grad_x=g)
            c.check_backward(g, grads, c.t64, _np(st).astype(np.float64), c.grad_addend)


@pytest.mark.parametrize("n,C", [(1, 1), (3, 5), (100, 64), (257, 65), (64, 96), (33, 250), (9, 512), (1000, 8)])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_checkpoint_store_and_load(env, n, C, x):
    dm, lib, torch = env
    announce("checkpoint", n, C, x)
    g = np.random.default_rng(n + C)
    v = g.normal(size=(n, C)) * np.exp(4 * g.normal(size=(n, 1)))
    t = torch.tensor(v, dtype=torch.float32, device="cuda").to({"f32": torch.float32, "bf16": torch.bfloat16}[x])
    if n > 8 and C >= 5:
        t[0] = 0.0
        t[1, C - 1] = float("inf")
        t[2, 0] = float("nan")
        t[3] = t[3] * 1e-38
        t[4, 0], t[4, 1:5] = 127.0, torch.tensor([0.5, 1.5, -2.5, 126.5], dtype=t.dtype, device="cuda")   # ties
        t[5] = -t[5].abs()
        t[6, 0] = float("-inf")
        t[7] = 3.0e38
    ck = lib.dsmp_checkpoint_store(t)
    q, scale = on.checkpoint(_np(t))
    assert np.array_equal(ck.q.cpu().numpy(), q)
    assert np.array_equal(ck.scale.cpu().numpy(), scale, equal_nan=True)
    want = on.values(q, scale)
    assert np.array_equal(_np(lib.dsmp_checkpoint_load(ck)), want, equal_nan=True)
    low = lib.dsmp_checkpoint_load(ck, torch.empty(n, C, dtype=torch.bfloat16, device="cuda"))
    assert np.array_equal(_np(low), _np(torch.tensor(want).to(torch.bfloat16)), equal_nan=True)


def test_infinities_and_nan_stay_in_their_segment_and_group(env):
    dm, lib, torch = env
    n, C, G = 600, 64, 4
    for segments in ([0, 200, 200, 450, 600], 600):
        for bad in (float("nan"), float("inf")):
            announce("norm non-finite", segments, bad)
            c = Case(torch, n, C, G, segments)
            clean, st0 = lib.dsmp_group_norm_forward(c.desc(dm), c.x, c.gamma, c.beta, segments=c.seg())
            x = c.x.clone()
            x[300, 20] = bad                       # second non-empty segment, group 1
            ck = dm.Checkpoint.empty(n, C, "cuda")
            y, st = lib.dsmp_group_norm_forward(c.desc(dm), x, c.gamma, c.beta, segments=c.seg(), checkpoint=ck)
            hit = torch.zeros(n, C, dtype=torch.bool, device="cuda")
            rows = slice(200, 450) if isinstance(segments, list) else slice(300, 301)
            hit[rows, 16:32] = True
            assert torch.equal(y[~hit], clean[~hit])
            assert torch.isnan(y[300, 20]) and not torch.isfinite(y[hit]).all()
            dx, grads = lib.dsmp_group_norm_backward(c.desc(dm), ck, st, c.gamma, c.beta, c.dy, segments=c.seg())
            block = hit.clone()
            block[300, :] = True                   # the row's checkpoint block is one scale
            rows_ok = ~block
            if isinstance(segments, list):         # its sums reach every group of the segment
                rows_ok[200:450] = False
            assert torch.isfinite(dx[rows_ok]).all() and torch.isnan(dx[300]).all()


def test_no_rows_and_empty_segments(env):
    dm, lib, torch = env
    announce("norm no rows")
    C, G = 32, 4
    d = dm.norm_desc(C, G, dm.F32, dm.F32, dm.ACT_SILU)
    x, dy = torch.empty(0, C, device="cuda"), torch.empty(0, C, device="cuda")
    gamma, beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    for seg, k in ((None, 1), (torch.zeros(4, dtype=torch.int32, device="cuda"), 3), (5, 5)):
        st = torch.full((k, G, 2), 9.0, device="cuda")
        ck = dm.Checkpoint.empty(0, C, "cuda")
        y, _ = lib.dsmp_group_norm_forward(d, x, gamma, beta, segments=seg, stats=st, checkpoint=ck)
        assert y.shape == (0, C) and (st == 0).all()
        lib.dsmp_group_norm_restore(d, ck, st, gamma, beta, segments=seg)
        grads = {"dgamma": torch.full((C,), 2.0, device="cuda"), "dbeta": torch.full((C,), 3.0, device="cuda")}
        lib.dsmp_group_norm_backward(d, ck, st, gamma, beta, dy, segments=seg, grads=grads, flags=dm.GRAD_ACCUMULATE)
        assert (grads["dgamma"] == 2).all() and (grads["dbeta"] == 3).all()
        lib.dsmp_group_norm_backward(d, x, st, gamma, beta, dy, segments=seg, grads=grads)
        assert (grads["dgamma"] == 0).all() and (grads["dbeta"] == 0).all()
    assert lib.dsmp_checkpoint_load(lib.dsmp_checkpoint_store(x)).shape == (0, C)


def test_gradients_accumulate(env):
    dm, lib, torch = env
    for segments in (None, 300):
        announce("norm accumulate", segments)
        c = Case(torch, 300, 40, 5, segments)
        d = c.desc(dm)
        _, st = lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=segments)
        dx, grads = lib.dsmp_group_norm_backward(d, c.x, st, c.gamma, c.beta, c.dy, segments=segments)
        lib.dsmp_group_norm_backward(d, c.x, st, c.gamma, c.beta, c.dy, segments=segments, grads=grads,
                                     flags=dm.GRAD_ACCUMULATE)
        c.check_backward(dx, grads, c.t64, _np(st).astype(np.float64), times=2)


def test_same_bits_on_every_run_and_on_another_stream(env):
    dm, lib, torch = env
    for segments in (None, [0, 5000, 5001, 30000], 30000):
        announce("norm determinism", segments)
        c = Case(torch, 30000, 64, 8, segments, "bf16", "bf16", on.GELU, addend=True)
        d, seg = c.desc(dm), c.seg()

        def go():
            ck = dm.Checkpoint.empty(c.n, c.C, "cuda")
            y, st = lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg, addend=c.addend,
                                                sum_out=torch.empty_like(c.x), checkpoint=ck)
            u = lib.dsmp_group_norm_restore(d, ck, st, c.gamma, c.beta, segments=seg)
            dx, gr = lib.dsmp_group_norm_backward(d, ck, st, c.gamma, c.beta, c.dy, segments=seg,
                                                  grad_addend=c.grad_addend)
            return [y, st, ck.q, ck.scale, u, dx, gr["dgamma"], gr["dbeta"]]

        first = go()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = go()
        second = go()
        torch.cuda.synchronize()
        for a, b, e in zip(first, second, other):
            assert torch.equal(bits(a), bits(b)) and torch.equal(bits(a), bits(e))


def test_replayed_from_a_graph(env):
    """A captured forward, restore and backward, replayed with new inputs and eager work between the replays."""
    dm, lib, torch = env
    for segments in (None, [0, 700, 2000], 2000):
        announce("norm graph", segments)
        c = Case(torch, 2000, 64, 8, segments, "f32", "bf16", addend=True)
        d, seg = c.desc(dm), c.seg()
        ck = dm.Checkpoint.empty(c.n, c.C, "cuda")
        b = {"sum": torch.empty_like(c.x), "y": torch.empty(c.n, c.C, dtype=torch.bfloat16, device="cuda"),
             "u": torch.empty(c.n, c.C, dtype=torch.bfloat16, device="cuda"), "dx": torch.empty(c.n, c.C, device="cuda"),
             "st": torch.empty(len(on.bounds(c.n, segments)) - 1, c.G, 2, device="cuda"),
             "dgamma": torch.empty(c.C, device="cuda"), "dbeta": torch.empty(c.C, device="cuda")}

        def go():
            lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg, addend=c.addend, sum_out=b["sum"],
                                        y=b["y"], stats=b["st"], checkpoint=ck)
            lib.dsmp_group_norm_restore(d, ck, b["st"], c.gamma, c.beta, segments=seg, y=b["u"])
            lib.dsmp_group_norm_backward(d, ck, b["st"], c.gamma, c.beta, c.dy, segments=seg, grad_x=b["dx"],
                                         grads={"dgamma": b["dgamma"], "dbeta": b["dbeta"]})

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            go()                                     # its scratch buffer exists before the capture
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            go()
        for k in range(4):
            c.x.copy_(torch.randn_like(c.x) + k)
            c.dy.copy_(torch.randn_like(c.dy))
            graph.replay()
            torch.cuda.synchronize()
            got = {n: v.clone() for n, v in b.items()}
            go()
            torch.cuda.synchronize()
            for n, v in b.items():
                assert torch.equal(bits(got[n]), bits(v)), (k, n)


def test_wrong_segment_bounds_write_nothing_outside(env):
    """Bounds that do not ascend, or leave the rows: limited on the device; the arrays' neighbours stay."""
    dm, lib, torch = env
    n, C, G = 500, 64, 8
    for segments in ([0, 400, 100, 500], [-7, 100, 9000, 20, 500], [500, 500, 0, 0], [0, 3, 2 ** 31 - 1, -2 ** 31, 4]):
        announce("norm wrong bounds", segments)
        c = Case(torch, n, C, G)
        seg = torch.tensor(segments, dtype=torch.int32, device="cuda")
        k = len(segments) - 1
        pad = 64
        y, dx = (torch.full((n + 2 * pad, C), 7.0, device="cuda") for _ in range(2))
        st = torch.full((k + 2, G, 2), 7.0, device="cuda")
        lib.dsmp_group_norm_forward(c.desc(dm), c.x, c.gamma, c.beta, segments=seg, y=y[pad:-pad], stats=st[1:-1])
        lib.dsmp_group_norm_backward(c.desc(dm), c.x, st[1:-1], c.gamma, c.beta, c.dy, segments=seg, grad_x=dx[pad:-pad])
        for t in (y[:pad], y[-pad:], dx[:pad], dx[-pad:], st[:1], st[-1:]):
            assert (t == 7).all()


def test_offsets_past_32_bits(env):
    """9.1 million rows of 256 channels: 2.3e9 values; the last segment against the oracle."""
    dm, lib, torch = env
    n, C, G, m = 9_100_000, 256, 32, 1000
    announce("norm large", n, C)
    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 60 GB")
    x = torch.empty(n, C, dtype=torch.bfloat16, device="cuda").normal_()
    c = Case(torch, m, C, G, None, "bf16", "bf16")
    x[n - m:] = c.x
    dy = torch.ones(n, C, device="cuda")
    dy[n - m:] = c.dy
    seg = torch.tensor([0, 5, n - m, n], dtype=torch.int32, device="cuda")
    ck = dm.Checkpoint.empty(n, C, "cuda")
    d = c.desc(dm)
    y, st = lib.dsmp_group_norm_forward(d, x, c.gamma, c.beta, segments=seg, checkpoint=ck)
    ref = c.check_stats(st[2:], c.t64)
    c.check_y(y[n - m:], c.t64, ref)
    q, scale = on.checkpoint(_np(c.x))
    assert np.array_equal(ck.q[n - m:].cpu().numpy(), q) and np.array_equal(ck.scale[n - m:].cpu().numpy(), scale)
    lib.dsmp_group_norm_restore(d, ck, st, c.gamma, c.beta, segments=seg, y=y)
    c.check_y(y[n - m:], on.values(q, scale).astype(np.float64), _np(st[2:]).astype(np.float64), "restored")
    del y
    dx, _ = lib.dsmp_group_norm_backward(d, x, st, c.gamma, c.beta, dy, segments=seg)
    c.gamma = None       # the parameters' gradients cover all rows: dx alone is compared
    c.check_backward(dx[n - m:], None, c.t64, _np(st[2:]).astype(np.float64))


def test_gradient_against_differences(env):
    """The library's own forward, stepped along random directions: central
    differences of sum(dy y) in float64.  With steps of 2^-6 on values of order
    one the third derivative leaves 1e-4 of the sum, rounding 4 u / 2^-6 of
    the terms' norm."""
    dm, lib, torch = env
    for segments in (None, [0, 50, 200], 200):
        announce("norm differences", segments)
        c = Case(torch, 200, 64, 8, segments, act=on.SILU, eps=1e-2)
        d, seg, h = c.desc(dm), c.seg(), 2.0 ** -6
        _, st = lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg)
        dx, grads = lib.dsmp_group_norm_backward(d, c.x, st, c.gamma, c.beta, c.dy, segments=seg)
        g = torch.Generator(device="cuda").manual_seed(3)

        def loss(x, gamma, beta):
            y, _ = lib.dsmp_group_norm_forward(d, x, gamma, beta, segments=seg)
            return float((y.double() * c.dy.double()).sum())

        for name, v, got in (("x", c.x, dx), ("gamma", c.gamma, grads["dgamma"]), ("beta", c.beta, grads["dbeta"])):
            e = torch.randn(v.shape, generator=g, device="cuda")
            args = {"x": c.x, "gamma": c.gamma, "beta": c.beta}
            up, dn = loss(**{**args, name: v + h * e}), loss(**{**args, name: v - h * e})
            want = float((got.double() * e.double()).sum())
            norm = float(got.double().norm()) * float(e.double().norm()) / e.numel() ** 0.5
            assert abs((up - dn) / (2 * h) - want) <= 5e-3 * norm, (name, (up - dn) / (2 * h), want)


def test_refusals(env):
    dm, lib, torch = env
    announce("norm refusals")
    n, C, G = 10, 32, 4
    x, f = torch.zeros(n, C, device="cuda"), torch.ones(C, device="cuda")
    ok = dm.norm_desc(C, G, dm.F32, dm.F32, dm.ACT_SILU)
    _, st = lib.dsmp_group_norm_forward(ok, x, f, f)
    ck = lib.dsmp_checkpoint_store(x)

    def refused(status, fn, *args, **kw):
        with pytest.raises(dm.DsmpError) as e:
            fn(*args, **kw)
        assert e.value.status == status, str(e.value)

    fwd, bwd, res = lib.dsmp_group_norm_forward, lib.dsmp_group_norm_backward, lib.dsmp_group_norm_restore
    wide = torch.zeros(n, 513, device="cuda")
    refused(dm.UNSUPPORTED, fwd, dm.norm_desc(513, 1, dm.F32, dm.F32), wide, None, None)
    refused(dm.UNSUPPORTED, lib.dsmp_checkpoint_store, wide)
    for d in (dm.norm_desc(C, 5, dm.F32, dm.F32), dm.norm_desc(C, 0, dm.F32, dm.F32),
              dm.norm_desc(C, G, dm.F32, dm.F32, 4), dm.norm_desc(C, G, dm.F32, dm.F32, 0, -1.0),
              dm.norm_desc(C, G, dm.F32, dm.F32, 0, float("nan")), dm.norm_desc(C, G, 2, dm.F32)):
        refused(dm.INVALID_ARG, fwd, d, x, f, f)
    refused(dm.INVALID_ARG, fwd, ok, x, f, None)                       # gamma without beta
    refused(dm.INVALID_ARG, fwd, ok, x, f, f, segments=3)              # 3 does not divide 10
    refused(dm.INVALID_ARG, fwd, ok, x, f, f, segments=0)
    refused(dm.INVALID_ARG, fwd, ok, x, f, f, addend=x)                # no place for the sum
    refused(dm.INVALID_ARG, fwd, ok, x.bfloat16(), f, f)
    refused(dm.INVALID_ARG, fwd, ok, x.cpu(), f, f)
    refused(dm.INVALID_ARG, fwd, ok, x.t(), f, f)
    refused(dm.INVALID_ARG, fwd, ok, torch.zeros(C, n, device="cuda").t(), f, f)
    refused(dm.INVALID_ARG, fwd, ok, torch.zeros(1, C, device="cuda").expand(n, C), f, f)
    refused(dm.INVALID_ARG, fwd, ok, x, f[:8], f)
    refused(dm.INVALID_ARG, fwd, ok, x, f, f, segments=torch.zeros(3, dtype=torch.int64, device="cuda"))
    refused(dm.INVALID_ARG, fwd, ok, x, f, f, stats=torch.zeros(1, G, 3, device="cuda"))
    refused(dm.INVALID_ARG, fwd, ok, x, f, f, checkpoint=dm.Checkpoint.empty(n, C + 1, "cuda"))
    refused(dm.INVALID_ARG, res, ok, dm.Checkpoint(ck.q, ck.scale[:5]), st, f, f)
    refused(dm.INVALID_ARG, bwd, ok, ck, st, f, f, x.bfloat16())
    refused(dm.INVALID_ARG, bwd, ok, ck, st[:, :2], f, f, x)
    refused(dm.INVALID_ARG, bwd, ok, ck, st, f, f, x, flags=dm.GRAD_X_ACCUMULATE)
    refused(dm.INVALID_ARG, lib.dsmp_checkpoint_store, x.half())
    refused(dm.INVALID_ARG, lib.dsmp_checkpoint_load, ck, torch.zeros(n, C, dtype=torch.float16, device="cuda"))
    # the layers take the first two activations alone
    desc = dm.layer_desc(2, 32, 64, 64, dm.F32, act=dm.ACT_SILU)
    g = lib.dsmp_radius_graph_build(torch.rand(n, 2, device="cuda"), n, 0.5)
    with pytest.raises(dm.DsmpError):
        lib.dsmp_nnconv_workspace(desc, g)


@pytest.mark.parametrize("C,G", [(96, 12), (40, 5), (33, 3), (512, 4)])
@pytest.mark.parametrize("segments", [None, [0, 10, 3000], 3000])
def test_sum_in_place_with_a_checkpoint(env, segments, C, G):
    """Widths at which a row's last lanes have no channels of their own, the sum written over x."""
    dm, lib, torch = env
    announce("norm in place, kept", segments, C)
    c = Case(torch, 3000, C, G, segments, "f32", "bf16", addend=True)
    x, ck = c.x.clone(), dm.Checkpoint.empty(3000, C, "cuda")
    y, st = lib.dsmp_group_norm_forward(c.desc(dm), x, c.gamma, c.beta, segments=c.seg(), addend=c.addend, sum_out=x,
                                        checkpoint=ck)
    assert torch.equal(x, c.t)
    c.check_y(y, c.t64, c.check_stats(st, c.t64))
    q, scale = on.checkpoint(_np(c.t))
    assert np.array_equal(ck.q.cpu().numpy(), q) and np.array_equal(ck.scale.cpu().numpy(), scale)


def test_refuses_rows_too_far_apart(env):
    dm, lib, torch = env
    announce("norm row distance")
    far = torch.zeros(2, (1 << 16) + 1, device="cuda")[:, :32]
    f = torch.ones(32, device="cuda")
    for call in (lambda: lib.dsmp_group_norm_forward(dm.norm_desc(32, 4, dm.F32, dm.F32), far, f, f),
                 lambda: lib.dsmp_checkpoint_store(far)):
        with pytest.raises(dm.DsmpError) as e:
            call()
        assert e.value.status == dm.UNSUPPORTED


def _many(n, count, seed):
    """count + 1 bounds of unequal segments, a fifth of them empty."""
    g = np.random.default_rng(seed)
    w = np.where(g.random(count) < 0.2, 0.0, g.exponential(size=count))
    return [0] + [int(v) for v in np.minimum(n, np.round(np.cumsum(w) / w.sum() * n))][:-1] + [n]


@pytest.mark.parametrize("n,C,G,segments", [(20000, 32, 4, 1000), (20000, 32, 4, _many(20000, 3001, 1)),
                                            (6001, 40, 5, _many(6001, 4200, 2)), (30000, 64, 8, _many(30000, 64, 3)),
                                            (30000, 64, 8, _many(30000, 65, 4)), (9999, 24, 2, 3333)])
def test_many_segments(env, n, C, G, segments):
    """More segments than a wave has lanes, and more pieces than there are workgroups."""
    dm, lib, torch = env
    announce("norm segments", n, C, len(segments) if isinstance(segments, list) else segments)
    c = Case(torch, n, C, G, segments, "f32", "f32", addend=True)
    d, seg = c.desc(dm), c.seg()
    ck, total = dm.Checkpoint.empty(n, C, "cuda"), torch.empty_like(c.x)
    y, st = lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg, addend=c.addend, sum_out=total,
                                        checkpoint=ck)
    c.check_y(y, c.t64, c.check_stats(st, c.t64))
    q, scale = on.checkpoint(_np(c.t))
    assert np.array_equal(ck.q.cpu().numpy(), q) and np.array_equal(ck.scale.cpu().numpy(), scale)
    st64, kept = _np(st).astype(np.float64), on.values(q, scale).astype(np.float64)
    c.check_y(lib.dsmp_group_norm_restore(d, ck, st, c.gamma, c.beta, segments=seg), kept, st64, "restored")
    dx, grads = lib.dsmp_group_norm_backward(d, ck, st, c.gamma, c.beta, c.dy, segments=seg, grad_addend=c.grad_addend)
    c.check_backward(dx, grads, kept, st64, c.grad_addend)


def test_refuses_statistics_between_pairs(env):
    dm, lib, torch = env
    announce("norm stats alignment")
    x, f = torch.zeros(10, 32, device="cuda"), torch.ones(32, device="cuda")
    d, st = dm.norm_desc(32, 4, dm.F32, dm.F32), torch.zeros(9, device="cuda")[1:].view(1, 4, 2)
    ck = lib.dsmp_checkpoint_store(x)
    for call in (lambda: lib.dsmp_group_norm_forward(d, x, f, f, stats=st),
                 lambda: lib.dsmp_group_norm_restore(d, ck, st, f, f),
                 lambda: lib.dsmp_group_norm_backward(d, ck, st, f, f, x)):
        with pytest.raises(dm.DsmpError) as e:
            call()
        assert e.value.status == dm.INVALID_ARG


@pytest.mark.parametrize("n", [511, 512, 513, 1024, 1025])
@pytest.mark.parametrize("segments", [None, 1, "two"])
def test_sizes_at_which_one_launch_becomes_two(env, n, segments):
    dm, lib, torch = env
    announce("norm one launch", n, segments)
    for add in (False, True):
        c = Case(torch, n, 32, 4, [0, n // 3, n] if segments == "two" else segments, addend=add)
        total, ck = (torch.empty_like(c.x), dm.Checkpoint.empty(n, 32, "cuda")) if add else (None, None)
        d, seg = c.desc(dm), c.seg()
        y, st = lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg, addend=c.addend, sum_out=total,
                                            checkpoint=ck)
        c.check_y(y, c.t64, c.check_stats(st, c.t64))
        dx, grads = lib.dsmp_group_norm_backward(d, c.t, st, c.gamma, c.beta, c.dy, segments=seg)
        c.check_backward(dx, grads, c.t64, _np(st).astype(np.float64))


def test_few_rows_in_millions_of_segments(env):
    dm, lib, torch = env
    announce("norm millions of segments")
    n, C, G, nseg = 10, 8, 2, (1 << 22) + 1   # 1,024 threads for each of them would be past 2^32
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn(n, C, device="cuda", generator=g) for _ in range(2))
    f = torch.full((C,), 1.5, device="cuda")
    ptr = torch.full((nseg + 1,), 3, dtype=torch.int32, device="cuda")   # rows 0..2 in the first, 3..9 in the last
    ptr[0], ptr[nseg] = 0, n
    two = torch.tensor([0, 3, n], dtype=torch.int32, device="cuda")
    d = dm.norm_desc(C, G, dm.F32, dm.F32, dm.ACT_SILU)
    y, st = lib.dsmp_group_norm_forward(d, x, f, f, segments=ptr)
    y2, st2 = lib.dsmp_group_norm_forward(d, x, f, f, segments=two)
    # the same formulas in another order of sums: a few units in the last place
    assert torch.allclose(st[[0, nseg - 1]], st2, rtol=32 * U, atol=32 * U) and torch.allclose(y, y2, rtol=0, atol=256 * U)
    assert not st[1:nseg - 1].any()
    dx, gr = lib.dsmp_group_norm_backward(d, x, st, f, f, dy, segments=ptr)
    dx2, gr2 = lib.dsmp_group_norm_backward(d, x, st2, f, f, dy, segments=two)
    assert torch.allclose(dx, dx2, rtol=0, atol=1024 * U)
    assert all(torch.allclose(gr[k], gr2[k], rtol=0, atol=1024 * U) for k in gr)


@pytest.mark.parametrize("n", [1, 7, 8, 9, 71, 72, 73, 700])
@pytest.mark.parametrize("C,G", [(1, 1), (3, 3), (5, 1), (9, 3), (13, 1), (30, 5), (66, 6), (129, 3), (263, 1)])
@pytest.mark.parametrize("rows", [False, True])
def test_rows_are_read_no_further_than_the_matrix(env, n, C, G, rows):
    # reads past a row's end stay in the matrix and never count: NaN between its rows, and it ends where
    # its buffer does
    dm, lib, torch = env
    announce("norm row ends", n, C, G, rows)
    for i, x in enumerate(("f32", "bf16")):
        c = Case(torch, n, C, G, n if rows else [0, n // 2, n], x, ("bf16", "f32")[i], on.SILU, addend=True, seed=i)
        d, seg = c.desc(dm), c.seg()

        def apart(t, gap):
            buf = torch.full(((n - 1) * (C + gap) + C,), float("nan"), dtype=t.dtype, device=t.device)
            m = buf.as_strided((n, C), (C + gap, 1))
            m.copy_(t)
            return m

        for gap in (0, 5):
            total, ck = apart(c.x, gap), dm.Checkpoint.empty(n, C, c.x.device)
            out, st = lib.dsmp_group_norm_forward(d, apart(c.x, gap), c.gamma, c.beta, segments=seg,
                                                  addend=apart(c.addend, gap), sum_out=total, checkpoint=ck)
            ref = c.check_stats(st, c.t64)
            assert torch.equal(total, c.t)
            c.check_y(out, c.t64, ref)
            q, scale = on.checkpoint(_np(c.t))
            assert np.array_equal(ck.q.cpu().numpy(), q) and np.array_equal(ck.scale.cpu().numpy(), scale)
            kept, st64 = on.values(q, scale), _np(st).astype(np.float64)
            c.check_y(lib.dsmp_group_norm_restore(d, ck, st, c.gamma, c.beta, segments=seg), kept, st64, "restored")
            dx, grads = lib.dsmp_group_norm_backward(d, total, st, c.gamma, c.beta, apart(c.dy, gap), segments=seg,
                                                     grad_addend=apart(c.grad_addend, gap))
            c.check_backward(dx, grads, c.t64, st64, c.grad_addend)
            again = lib.dsmp_checkpoint_store(apart(c.t, gap))
            assert torch.equal(again.q, ck.q) and torch.equal(again.scale, ck.scale)


@pytest.mark.parametrize("act", [on.RELU, on.IDENTITY])
@pytest.mark.parametrize("n,C,G", [(300, 64, 4), (3000, 64, 4), (100, 160, 5), (3000, 160, 5), (3000, 33, 3), (200, 33, 3)])
def test_an_infinity_leaves_no_number_in_its_group(env, n, C, G, act):
    """x - mean and the variance of a group with an infinity are no numbers: neither is its rstd, nor any of its
    results, whatever the place of the infinity and however its rows are joined."""
    dm, lib, torch = env
    c = C // G
    for segments in (None, [0, n // 3, n // 3, n], n):
        for bad in (float("inf"), -float("inf")):
            k = Case(torch, n, C, G, segments, act=act)
            clean, st0 = lib.dsmp_group_norm_forward(k.desc(dm), k.x, k.gamma, k.beta, segments=k.seg())
            b = on.bounds(n, segments)
            for i in (0, n // 3, n // 2, n - 1):
                announce("norm infinity", n, C, G, act, segments, bad, i)
                x = k.x.clone()
                x[i, c + 1] = bad                                        # group 1
                y, st = lib.dsmp_group_norm_forward(k.desc(dm), x, k.gamma, k.beta, segments=k.seg())
                s = int(np.searchsorted(b, i, side="right")) - 1         # the segment that has the row
                assert not torch.isfinite(st[s, 1, 0]) and torch.isnan(st[s, 1, 1])
                hit = torch.zeros(n, C, dtype=torch.bool, device="cuda")
                hit[b[s]:b[s + 1], c:2 * c] = True
                assert torch.isnan(y[hit]).all() and torch.equal(y[~hit], clean[~hit])
                other = torch.ones(st.shape[:2], dtype=torch.bool, device="cuda")
                other[s, 1] = False
                assert torch.equal(st[other], st0[other])


def test_rows_gradients_of_the_parameters_join_in_more_than_32_bits(env):
    """Each row a segment: the sums of a workgroup's four waves, 2^26, 1, 1 and -2^26, give 2 (in float32, 0)."""
    dm, lib, torch = env
    announce("norm rows, joined sums")
    n, C = 32, 32                                   # eight rows to a wave
    g = np.random.default_rng(1)
    x = torch.tensor(g.normal(size=(n, C)), dtype=torch.float32, device="cuda")
    x[24] = x[0]
    f, dy = torch.ones(C, device="cuda"), torch.zeros(n, C, device="cuda")
    for row, v in ((0, 2.0 ** 26), (8, 1.0), (16, 1.0), (24, -2.0 ** 26)):
        dy[row] = v
    d = dm.norm_desc(C, 4, dm.F32, dm.F32, dm.ACT_IDENTITY)
    _, st = lib.dsmp_group_norm_forward(d, x, f, 0 * f, segments=n)
    _, grads = lib.dsmp_group_norm_backward(d, x, st, f, 0 * f, dy, segments=n)
    assert (grads["dbeta"] == 2).all()
    xn = on.normalised(_np(x), _np(st).astype(np.float64), n)
    # the two large terms are equal and opposite; what is left is two values' own roundings
    assert (np.abs(_np(grads["dgamma"]) - (xn[8] + xn[16])) <= 16 * U * (1 + np.abs(xn[8]) + np.abs(xn[16]))).all()


def _gelu(z):
    """GELU and its slope, with the tail's own digits."""
    z = np.asarray(z, np.float64)
    tail = np.array([0.5 * math.erfc(abs(v) / math.sqrt(2.0)) for v in z.ravel()]).reshape(z.shape)
    phi = np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return np.where(z < 0, z * tail, z * (1 - tail)), np.where(z < 0, tail, 1 - tail) + z * phi, tail, phi


def test_gelu_keeps_the_digits_of_its_tail(env):
    """GELU and its slope at chosen arguments (mean 0, rstd 1), relative to their size.

    The tail: 3 u of the polynomial, 1 of its coefficients, 3 of its argument times at most 2.6 (how much
    faster than the argument it changes), 6 of the evaluation, products and the exponential, and 1.2 z^2 u of
    the exponent's roundings; with 10 % to spare below (20 + 1.5 z^2) u."""
    dm, lib, torch = env
    announce("norm GELU tail")
    n, C = 50, 256
    q = torch.arange(n * C, device="cuda").view(n, C) % 255 - 127
    scale = torch.linspace(0.001, 12.4 / 127, n * 4, device="cuda").view(n, 4)
    ck = dm.Checkpoint(q.to(torch.int8), scale)
    z = _np(ck.q.float() * scale.repeat_interleave(64, 1)).astype(np.float64)
    want, slope, tail, phi = _gelu(z)
    rel = (20 + 1.5 * z * z) * U
    for segments in (None, n):
        for C2, G in ((C, 4), (250, 5)):           # whole groups of four channels, and others
            part = dm.Checkpoint(ck.q[:, :C2].contiguous(), scale)
            st = torch.zeros(n if segments else 1, G, 2, device="cuda")
            st[:, :, 1] = 1.0
            y = lib.dsmp_group_norm_restore(dm.norm_desc(C2, G, dm.F32, dm.F32, dm.ACT_GELU), part, st, None, None,
                                            segments=segments)
            ref, zz = want[:, :C2], z[:, :C2]
            tol = np.abs(zz) * tail[:, :C2] * rel[:, :C2] + 3 * U * np.abs(ref) + 1e-37
            err = np.abs(_np(y).astype(np.float64) - ref)
            assert (err <= tol).all(), float((err / tol).max())
    # a row by itself: dbeta is the slope at each of its arguments
    f = torch.ones(C, device="cuda")
    st = torch.tensor([0.0, 1.0], device="cuda").expand(1, 4, 2).contiguous()
    d = dm.norm_desc(C, 4, dm.F32, dm.F32, dm.ACT_GELU)
    for i in range(n):
        row = dm.Checkpoint(ck.q[i:i + 1].contiguous(), scale[i:i + 1].contiguous())
        _, grads = lib.dsmp_group_norm_backward(d, row, st, f, 0 * f, torch.ones(1, C, device="cuda"))
        tol = (tail[i] + np.abs(z[i]) * phi[i]) * rel[i] + 3 * U * np.abs(slope[i]) + 1e-36
        err = np.abs(_np(grads["dbeta"]).astype(np.float64) - slope[i])
        assert (err <= tol).all(), (i, float((err / tol).max()))


@pytest.mark.parametrize("own", [False, True])
def test_a_graph_keeps_its_scratch_to_itself(env, own):
    """Captured calls, then a larger eager call on the capturing stream and new tensors there, then replays: the graph
    writes nothing of theirs and gives what eager calls do, beside eager work on the capturing stream too."""
    dm, lib, torch = env
    announce("norm graph scratch", own)
    n, C, G = 30000, 64, 8
    c = Case(torch, n, C, G, [0, 9000, n], "f32", "f32")
    d, seg = c.desc(dm), c.seg()
    big = Case(torch, 80000, 256, 64)
    b = {"y": torch.empty_like(c.x), "st": torch.empty(2, G, 2, device="cuda"), "dx": torch.empty_like(c.x),
         "dgamma": torch.empty(C, device="cuda"), "dbeta": torch.empty(C, device="cuda")}
    ws = torch.empty(max(lib.dsmp_group_norm_workspace(d, n, seg)), dtype=torch.uint8, device="cuda") if own else None

    def go(out, ws=None):
        lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg, y=out["y"], stats=out["st"], ws=ws)
        lib.dsmp_group_norm_backward(d, c.x, out["st"], c.gamma, c.beta, c.dy, segments=seg, grad_x=out["dx"],
                                     grads={"dgamma": out["dgamma"], "dbeta": out["dbeta"]}, ws=ws)

    want = {k: torch.empty_like(v) for k, v in b.items()}
    go(want)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        go({k: torch.empty_like(v) for k, v in b.items()})        # the stream has a scratch buffer
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        go(b, ws)
    big_desc = big.desc(dm)
    big_y, big_st = lib.dsmp_group_norm_forward(big_desc, big.x, big.gamma, big.beta)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        lib.dsmp_group_norm_forward(big_desc, big.x, big.gamma, big.beta)     # needs a larger one
        new = [torch.full((size,), 7, dtype=torch.uint8, device="cuda")
               for size in (1 << 9, 1 << 12, 1 << 16, 1 << 18, 1 << 20, 1 << 21) for _ in range(8)]
    torch.cuda.synchronize()
    for _ in range(3):
        for v in b.values():
            v.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            y, st = lib.dsmp_group_norm_forward(big_desc, big.x, big.gamma, big.beta)
        graph.replay()                                            # on the current stream, beside that call
        torch.cuda.synchronize()
        assert torch.equal(y, big_y) and torch.equal(st, big_st)
        for k in b:
            assert torch.equal(bits(b[k]), bits(want[k])), k
        assert all((t == 7).all() for t in new)


@pytest.mark.parametrize("C,G", [(32, 4), (128, 32), (100, 10), (147, 7), (512, 512), (1, 1)])
@pytest.mark.parametrize("n,segments", [(1, None), (37, 37), (700, [0, 0, 71, 700, 700]), (40000, None), (40000, 4000),
                                        (5000, "many")])
def test_calls_stay_within_a_workspace_of_the_reported_size(env, n, segments, C, G):
    dm, lib, torch = env
    announce("norm workspace", n, C, G, segments)
    segments = _many(n, 2500, 7) if segments == "many" else segments
    guard = 4096
    for x in ("f32", "bf16"):
        c = Case(torch, n, C, G, segments, x, "f32")
        d, seg = c.desc(dm), c.seg()
        sizes = lib.dsmp_group_norm_workspace(d, n, seg)
        y0, st0 = lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg)
        dx0, g0 = lib.dsmp_group_norm_backward(d, c.x, st0, c.gamma, c.beta, c.dy, segments=seg)

        def within(size, call):
            buf = torch.full((size + 2 * guard,), 0xAB, dtype=torch.uint8, device="cuda")
            out = call(buf[guard:guard + size])
            assert (buf[:guard] == 0xAB).all() and (buf[guard + size:] == 0xAB).all()
            return out

        y, st = within(sizes[0], lambda ws: lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg, ws=ws))
        dx, g = within(sizes[1], lambda ws: lib.dsmp_group_norm_backward(d, c.x, st, c.gamma, c.beta, c.dy,
                                                                         segments=seg, ws=ws))
        for u, v in ((y, y0), (st, st0), (dx, dx0), (g["dgamma"], g0["dgamma"]), (g["dbeta"], g0["dbeta"])):
            assert torch.equal(bits(u), bits(v))
        for size, call in ((sizes[0], lambda ws: lib.dsmp_group_norm_forward(d, c.x, c.gamma, c.beta, segments=seg, ws=ws)),
                           (sizes[1], lambda ws: lib.dsmp_group_norm_backward(d, c.x, st, c.gamma, c.beta, c.dy,
                                                                              segments=seg, ws=ws))):
            if size:
                with pytest.raises(dm.DsmpError) as e:
                    call(torch.empty(size - 1, dtype=torch.uint8, device="cuda"))
                assert e.value.status == dm.WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("n,C,G", [(300, 32, 2), (20000, 32, 2), (20000, 33, 3), (60000, 64, 1)])
def test_statistics_and_results_far_from_zero(env, n, C, G, x):
    """Values at 1e3 and 1e5 times their deviation, whose means are float32 values.

    Mean: 8 u |mean|.  A tile adds 16 values one by one, 1.4 u |mean| rms, before that averages out over
    tiles; a row's 64 channels give 0.6 u rms; six times that, a join and the kept mean's own rounding.
    rstd: squares are taken about the means of tiles, so an error `off` of a mean, in deviations, adds
    off^2; it also meets the tile's own distance from the mean, a quarter of a deviation for 16 values,
    which averages out over the N tiles: six deviations of that, off / 4 * 6 / sqrt N, at most off / 4.  Its
    own sums: 32 u."""
    dm, lib, torch = env
    for offset in (1e3, 1e5):
        for segments in (None, [0, n // 3, n], n):
            announce("norm far from zero", n, C, G, x, offset, segments)
            c = Case(torch, n, C, G, segments, x, "f32", on.IDENTITY, offset=0.0, affine=False)
            if x == "bf16":       # whole steps of bfloat16's spacing there
                step = 2.0 ** (math.floor(math.log2(offset)) - 7)
                c.x = (c.x.float().clamp(-20, 20).round() * step + math.floor(offset / step) * step).bfloat16()
            else:
                c.x = c.x + offset
            t64, per = _np(c.x).astype(np.float64), C // G
            y, st = lib.dsmp_group_norm_forward(c.desc(dm), c.x, None, None, segments=c.seg())
            if segments == n:
                v = t64.reshape(n, G, per)
                mean, tiles = v.mean(2), 1
                ref = np.stack([mean, 1 / np.sqrt(((v - mean[:, :, None]) ** 2).mean(2) + c.eps)], -1)
            else:
                ref, tiles = on.statistics(t64, segments, G, c.eps), n // 3 * per / 16
            got = _np(st).astype(np.float64)
            emean = 8 * U * np.abs(t64).max()
            assert (np.abs(got[:, :, 0] - ref[:, :, 0]) <= emean).all()
            off = emean * ref[:, :, 1]
            tol = off * off + off / 4 * min(1.0, 6 / math.sqrt(tiles)) + 32 * U
            far = np.abs(got[:, :, 1] / ref[:, :, 1] - 1)
            assert (far <= tol).all(), float((far / tol).max())
            xn = on.normalised(t64, ref, segments)
            row = np.repeat(np.arange(len(ref)), np.diff(on.bounds(n, segments)))
            most = np.repeat(off[row], per, 1) + np.abs(xn) * (np.repeat(tol[row], per, 1) + 8 * U) + 2 * U
            assert (np.abs(_np(y).astype(np.float64) - xn) <= most).all()
