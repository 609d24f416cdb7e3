"""Cases of the normalisation and checkpoint operators: what a program that trains
or runs a deep stack of message-passing layers does between the layers.

A pre-norm residual stack normalises its node features (rows of C channels,
channels last) over groups of channels, within each packed sub-graph or within
each row, applies an activation and hands the result to the next layer.  For
training it keeps the normalised input in 8 bits, rebuilds the layer's operand
from it in the backward pass, and takes the norm's gradients from it.

Sizes are those of the repository's workloads and their neighbours: about a
thousand nodes (a sampled 64 x 64 grid) to 285,564 (a channel slab with its halo
rows), widths 32 to 256.  Node features have offsets and scales of their own for
each channel, and a few values far out.
"""

import math

import torch

own = False

EPS = 1e-5
BLOCK = 64          # channels that share a checkpoint scale
TINY = 2.0 ** -100  # blocks whose largest value is below this are kept as zeros


def listed():
    return [
        # evaluation of a small sampled square: the smallest call (latency)
        dict(name="forward-1k", kind="forward", n=1024, C=32, G=8, x="f32", y="f32", act="silu", segs=1, addend=False),
        # evaluation of 37 sub-domains of one domain packed one after another, an odd number of nodes, two of them empty
        dict(name="forward-packed-100k", kind="forward", n=99991, C=64, G=16, x="bf16", y="bf16", act="gelu", segs=37,
             addend=False),
        # forward pass of a training step on a channel slab: float32 residual stream, the layer's output added on the way
        dict(name="forward-262k", kind="forward", n=262144, C=128, G=32, x="f32", y="bf16", act="silu", segs=1,
             addend=True),
        # each node normalised by itself (statistics of one row)
        dict(name="forward-rows-8k", kind="forward", n=8192, C=64, G=1, x="bf16", y="bf16", act="silu", segs=-1,
             addend=False),
        # training step of the operator on a small square: forward with checkpoint, restored operand, backward
        dict(name="train-1k", kind="train", n=1000, C=32, G=4, x="f32", y="f32", act="silu", segs=1, addend=True),
        # the same for eight packed sub-domains of an airfoil-like mesh, bf16 stream
        dict(name="train-packed-33k", kind="train", n=32768, C=64, G=8, x="bf16", y="bf16", act="gelu", segs=8,
             addend=True),
        # the largest: a channel slab with halo rows, float32 residual stream, bf16 operands of the layers
        dict(name="train-286k", kind="train", n=285564, C=128, G=32, x="f32", y="bf16", act="silu", segs=1,
             addend=True),
        # backward from the full-precision input, a 2-D square
        dict(name="backward-8k", kind="backward", n=8192, C=64, G=8, x="bf16", y="bf16", act="gelu", segs=1,
             addend=False),
        # backward of a per-node norm on a long channel, from the full-precision input
        dict(name="backward-rows-100k", kind="backward", n=100000, C=128, G=8, x="f32", y="f32", act="silu", segs=-1,
             addend=True),
        # the layers' operand rebuilt from the checkpoint, large slab
        dict(name="restore-262k", kind="restore", n=262144, C=128, G=32, x="f32", y="bf16", act="silu", segs=1,
             addend=False),
        # any activation kept in 8 bits and read back: a ragged width
        dict(name="checkpoint-8k", kind="checkpoint", n=8191, C=96, G=1, x="bf16", y="bf16", act="identity", segs=1,
             addend=False),
        # the same at the width of the largest kernel network
        dict(name="checkpoint-100k", kind="checkpoint", n=100000, C=256, G=1, x="f32", y="bf16", act="identity", segs=1,
             addend=False),
    ]


LARGEST = 285564 * 128
KINDS = ["forward", "train", "backward", "restore", "checkpoint"]


def draw(rng):
    kind = rng.choice(KINDS)
    # widths of the layers, and others a node network may have: odd counts of 8 among them, and some of none
    C = rng.choice([32, 64, 128, 256, rng.randrange(8, 257), 8 * rng.randrange(1, 33)])
    x = rng.choice(["f32", "bf16"])
    y = rng.choice(["f32", "bf16"])
    act = rng.choice(["identity", "silu", "gelu"])
    segs = rng.choice([1, 1, -1, max(2, round(math.exp(rng.uniform(math.log(2), math.log(96)))))])
    # groups of at least eight channels (the whole row where its width has no such divisor)
    G = rng.choice([g for g in range(1, C + 1) if C % g == 0 and C // g >= 8])
    most = min(286000, LARGEST // C)
    n = max(1, min(most, round(math.exp(rng.uniform(0.0, math.log(most + 1))))))
    if kind == "train":
        n = max(n, 16)
    if n == 3 * 1024:
        n += 1
    if segs > 1:
        segs = max(2, min(segs, 2 + n // 16))
    return dict(kind=kind, n=n, C=C, G=G, x=x, y=y, act=act, segs=segs, addend=rng.random() < 0.5)


DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def segment_ends(n, segs):
    """Where the packed segments begin and end: of unequal lengths, and from the third on some of none."""
    if segs == 1:
        return [0, n]
    w = [0.0 if (i % 17) == 3 else 0.25 + ((i * 0.6180339887) % 1.0) * 2.0 for i in range(segs)]
    total, at, ends = sum(w), 0.0, [0]
    for v in w:
        at += v
        ends.append(min(n, int(round(n * at / total))))
    ends[-1] = n
    return ends


def quantise(t):
    """(q, scale) of float32 rows: blocks of 64 channels, the last one shorter."""
    n, C = t.shape
    nb = (C + BLOCK - 1) // BLOCK
    pad = torch.zeros(n, nb * BLOCK - C, device=t.device)
    b = torch.cat([t, pad], 1).view(n, nb, BLOCK)
    a = b.abs().amax(2)
    some = a >= TINY
    scale = torch.where(some, a * torch.tensor(1.0 / 127.0, device=t.device), torch.zeros_like(a))
    inv = torch.where(some, torch.full_like(a, 127.0) / a, torch.zeros_like(a))
    q = torch.round(b * inv[:, :, None]).clamp(-127, 127)
    return q.view(n, nb * BLOCK)[:, :C].to(torch.int8).contiguous(), scale


def values(q, scale):
    """The float32 values that a checkpoint stands for."""
    n, C = q.shape
    return q.float() * scale.repeat_interleave(BLOCK, 1)[:, :C]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    n, C, G = case["n"], case["C"], case["G"]
    kind, xd, yd = case["kind"], DTYPES[case["x"]], DTYPES[case["y"]]
    f32 = dict(device=dev, dtype=torch.float32)

    def normal(*shape):
        return torch.randn(*shape, generator=g, **f32)

    x = normal(n, C) * torch.exp(0.4 * normal(C)) + normal(C)
    x = torch.where(torch.rand(n, C, generator=g, **f32) < 2e-4, 12.0 * x, x)
    s = dict(case=case, C=C, n=n, seg=None, xd=xd, yd=yd)
    if case["segs"] > 1:
        s["seg"] = torch.tensor(segment_ends(n, case["segs"]), dtype=torch.int32, device=dev)
    s["gamma"] = 1.0 + 0.2 * normal(C)
    s["beta"] = 0.2 * normal(C)
    segs = n if case["segs"] == -1 else case["segs"]
    if kind in ("forward", "train", "checkpoint"):
        s["x"] = x.to(xd)
    if kind in ("forward", "train"):
        s["addend"] = (0.5 * normal(n, C)).to(xd) if case["addend"] else None
        s["sum"] = torch.empty(n, C, device=dev, dtype=xd) if case["addend"] else None
        s["stats"] = torch.empty(segs, G, 2, **f32)
    if kind in ("backward", "restore"):
        x = x.to(xd).float()
        mean, var = statistics(x, s["seg"], segs, G)
        s["stats"] = torch.stack([mean, torch.rsqrt(var + EPS)], -1).contiguous()
        if kind == "backward":
            s["x"] = x.to(xd)
        else:
            s["q"], s["scale"] = quantise(x)
    if kind in ("train", "backward"):
        s["dy"] = normal(n, C)
        s["grad_addend"] = normal(n, C) if case["addend"] else None
        s["dx"] = torch.empty(n, C, **f32)
        s["dgamma"], s["dbeta"] = torch.empty(C, **f32), torch.empty(C, **f32)
    if kind in ("train", "checkpoint"):
        s["q"] = torch.empty(n, C, device=dev, dtype=torch.int8)
        s["scale"] = torch.empty(n, (C + BLOCK - 1) // BLOCK, **f32)
    if kind != "backward":
        s["y"] = torch.empty(n, C, device=dev, dtype=yd)
    if kind == "train":
        s["u"] = torch.empty(n, C, device=dev, dtype=yd)
    return s


# ---------------------------------------------------------------- plain form

def membership(seg, n):
    """float32 [segments, n]: 1 where a row belongs to a segment."""
    row = torch.arange(n, device=seg.device, dtype=torch.int32)
    return ((row >= seg[:-1, None]) & (row < seg[1:, None])).float()


def per_segment(v, seg, segs):
    """Sums [segments, G] of the row values [n, G]."""
    n = v.shape[0]
    if segs == n:
        return v
    return v.sum(0, keepdim=True) if seg is None else membership(seg, n) @ v


def to_rows(v, seg, segs, n):
    """The row of its segment for each of n rows."""
    if segs == n:
        return v
    if seg is None:
        return v.expand(n, v.shape[1])
    row = torch.arange(n, device=v.device, dtype=torch.int32)
    return v[torch.searchsorted(seg[1:].contiguous(), row, right=True)]


def counts(seg, segs, n, c, dev):
    """Values of each segment's group [segments, 1]."""
    if seg is None:
        return torch.full((segs, 1), float(n // segs * c), device=dev)
    return (seg[1:] - seg[:-1]).float()[:, None] * c


def statistics(x, seg, segs, G):
    """(mean, variance) [segments, G] of float32 rows; zero where a segment is empty."""
    n, C = x.shape
    m = counts(seg, segs, n, C // G, x.device).clamp(min=1.0)
    mean = per_segment(x.view(n, G, C // G).sum(2), seg, segs) / m
    off = x.view(n, G, C // G) - to_rows(mean, seg, segs, n)[:, :, None]
    return mean, per_segment((off * off).sum(2), seg, segs) / m


def activated(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def slope(z, act):
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return torch.ones_like(z)


def normalised(x, stats, seg, segs):
    n, C = x.shape
    G = stats.shape[1]
    mean, rstd = to_rows(stats[:, :, 0], seg, segs, n), to_rows(stats[:, :, 1], seg, segs, n)
    return ((x.view(n, G, C // G) - mean[:, :, None]) * rstd[:, :, None]).view(n, C)


def plain_forward(s, segs, G):
    x = s["x"].float()
    out = {}
    if s["addend"] is not None:
        out["sum"] = (x + s["addend"].float()).to(s["xd"])
        x = out["sum"].float()
    mean, var = statistics(x, s["seg"], segs, G)
    rstd = 1.0 / torch.sqrt(var + EPS)
    if s["seg"] is not None:
        rstd = torch.where((s["seg"][1:] > s["seg"][:-1])[:, None], rstd, torch.zeros_like(rstd))
    out["stats"] = torch.stack([mean, rstd], -1)
    z = normalised(x, out["stats"], s["seg"], segs) * s["gamma"] + s["beta"]
    out["y"] = activated(z, s["case"]["act"]).to(s["yd"])
    return out, x


def plain_backward(s, x, stats, segs, G):
    n, C = x.shape
    c, seg = C // G, s["seg"]
    xn = normalised(x, stats, seg, segs)
    w = s["dy"] * slope(xn * s["gamma"] + s["beta"], s["case"]["act"])
    m = counts(seg, segs, n, c, x.device).clamp(min=1.0)
    gw = w * s["gamma"]
    a = to_rows(per_segment(gw.view(n, G, c).sum(2), seg, segs) / m, seg, segs, n)[:, :, None]
    b = to_rows(per_segment((gw * xn).view(n, G, c).sum(2), seg, segs) / m, seg, segs, n)[:, :, None]
    rstd = to_rows(stats[:, :, 1], seg, segs, n)[:, :, None]
    dx = (rstd * (gw.view(n, G, c) - a - xn.view(n, G, c) * b)).view(n, C)
    if s["grad_addend"] is not None:
        dx = dx + s["grad_addend"]
    return {"dx": dx, "dgamma": (w * xn).sum(0), "dbeta": w.sum(0)}


def plain(s):
    case = s["case"]
    kind, G = case["kind"], case["G"]
    segs = s["n"] if case["segs"] == -1 else case["segs"]
    if kind == "checkpoint":
        return {"values": values(*quantise(s["x"].float())).to(s["yd"])}
    if kind == "backward":
        return plain_backward(s, s["x"].float(), s["stats"], segs, G)
    if kind == "restore":
        z = normalised(values(s["q"], s["scale"]), s["stats"], s["seg"], segs) * s["gamma"] + s["beta"]
        return {"u": activated(z, case["act"]).to(s["yd"])}
    out, x = plain_forward(s, segs, G)
    if kind == "train":
        v = values(*quantise(x))
        z = normalised(v, out["stats"], s["seg"], segs) * s["gamma"] + s["beta"]
        out["u"] = activated(z, case["act"]).to(s["yd"])
        out.update(plain_backward(s, v, out["stats"], segs, G))
    return out


# ------------------------------------------------------------ the framework's

_handle = []


def kernels(s):
    import paper_2402_15106_amd as dm
    if not _handle:
        _handle.append(dm.Dsmp(0))
    lib, case = _handle[0], s["case"]
    kind = case["kind"]
    if kind == "checkpoint":
        ck = lib.dsmp_checkpoint_store(s["x"], out=dm.Checkpoint(s["q"], s["scale"]))
        return {"values": lib.dsmp_checkpoint_load(ck, s["y"])}
    act = {"identity": dm.ACT_IDENTITY, "silu": dm.ACT_SILU, "gelu": dm.ACT_GELU}[case["act"]]
    code = {"f32": dm.F32, "bf16": dm.BF16}
    desc = dm.norm_desc(s["C"], case["G"], code[case["x"]], code[case["y"]], act, EPS)
    seg = s["n"] if case["segs"] == -1 else s["seg"]
    gamma, beta = s["gamma"], s["beta"]
    if kind == "restore":
        return {"u": lib.dsmp_group_norm_restore(desc, dm.Checkpoint(s["q"], s["scale"]), s["stats"], gamma, beta,
                                                 segments=seg, y=s["y"])}
    out, src = {}, s.get("x")
    if kind in ("forward", "train"):
        src = dm.Checkpoint(s["q"], s["scale"]) if kind == "train" else None
        out["y"], out["stats"] = lib.dsmp_group_norm_forward(desc, s["x"], gamma, beta, segments=seg,
                                                             addend=s["addend"], sum_out=s["sum"], y=s["y"],
                                                             stats=s["stats"], checkpoint=src)
        if s["sum"] is not None:
            out["sum"] = s["sum"]
    if kind == "train":
        out["u"] = lib.dsmp_group_norm_restore(desc, src, s["stats"], gamma, beta, segments=seg, y=s["u"])
    if kind in ("train", "backward"):
        out["dx"], grads = lib.dsmp_group_norm_backward(desc, src, s["stats"], gamma, beta, s["dy"], segments=seg,
                                                        grad_addend=s["grad_addend"], grad_x=s["dx"],
                                                        grads={"dgamma": s["dgamma"], "dbeta": s["dbeta"]})
        out.update(grads)
    return out


def run(state):
    return kernels(state) if own else plain(state)


def work(case):
    n, C, kind = case["n"], case["C"], case["kind"]
    size = {"f32": 4, "bf16": 2}
    xb, yb = size[case["x"]], size[case["y"]]
    el = n * C
    segs = n if case["segs"] == -1 else case["segs"]
    kept = el + 4 * n * ((C + BLOCK - 1) // BLOCK)      # a checkpoint's bytes
    stats, params = 8 * segs * case["G"], 8 * C
    if kind == "checkpoint":
        return {"bytes": el * (xb + yb) + 2 * kept, "flops": 4 * el}
    if kind == "restore":
        return {"bytes": el * yb + kept + stats + params, "flops": 10 * el}
    forward = el * (xb + yb + (2 * xb if case["addend"] else 0)) + stats + params
    backward = el * (8 + (4 if case["addend"] else 0)) + stats + 2 * params
    if kind == "forward":
        return {"bytes": forward, "flops": 12 * el}
    if kind == "backward":
        return {"bytes": backward + el * xb, "flops": 30 * el}
    # the checkpoint is written by the forward pass and read by the restored operand and the backward pass
    return {"bytes": forward + 3 * kept + el * yb + stats + params + backward, "flops": 56 * el}


# ------------------------------------------------------------ 64 bits

def exact(case, seed):
    """The same from the definitions in 64 bits, one segment at a time."""
    n, C, G, kind = case["n"], case["C"], case["G"], case["kind"]
    c = C // G
    s = prepare(case, seed)
    d = torch.float64

    def rounded64(v):
        """What an 8-bit checkpoint of float64 rows stands for."""
        out = torch.zeros_like(v)
        for k in range(0, C, BLOCK):
            b = v[:, k:k + BLOCK]
            unit = b.abs().max(1, keepdim=True).values / 127.0
            out[:, k:k + BLOCK] = torch.where(unit > 0, torch.round(b / unit.clamp(min=1e-300)) * unit, unit)
        return out

    def act64(z, want_slope):
        if case["act"] == "identity":
            return torch.ones_like(z) if want_slope else z
        if case["act"] == "silu":
            p = torch.sigmoid(z)
            return p + z * p * (1.0 - p) if want_slope else z * p
        phi = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return phi + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi) if want_slope else z * phi

    if kind == "checkpoint":
        return {"values": rounded64(s["x"].to(d))}
    gamma, beta = s["gamma"].to(d), s["beta"].to(d)
    rows = case["segs"] == -1
    ends = None if rows else segment_ends(n, max(1, case["segs"]))

    def pieces():
        """Every segment's rows as [instances, rows, C]: all rows at once where each is an instance."""
        if rows:
            yield slice(0, n), slice(0, n), (n, 1)
            return
        for i in range(len(ends) - 1):
            if ends[i + 1] > ends[i]:
                yield slice(i, i + 1), slice(ends[i], ends[i + 1]), (1, ends[i + 1] - ends[i])

    out = {}
    if kind in ("forward", "train"):
        t = s["x"].to(d)
        if s["addend"] is not None:
            out["sum"] = t + s["addend"].to(d)
            t = out["sum"].to(s["xd"]).to(d)        # the stream's own values are what is normalised
    elif kind == "backward":
        t = s["x"].to(d)
    else:
        wide = s["scale"].to(d).repeat_interleave(BLOCK, 1)[:, :C]
        t = s["q"].to(d) * wide
    kept = None
    if kind == "train":
        q, scale = quantise(t.float())               # the checkpoint itself is whole numbers and 32-bit scales
        kept = q.to(d) * scale.to(d).repeat_interleave(BLOCK, 1)[:, :C]
    stats = torch.zeros(n if rows else len(ends) - 1, G, 2, dtype=d, device=t.device)
    res = {k: torch.zeros(n, C, dtype=d, device=t.device) for k in ("y", "u", "dx")}
    dgamma, dbeta = torch.zeros(C, dtype=d, device=t.device), torch.zeros(C, dtype=d, device=t.device)
    for which, at, (inst, r) in pieces():
        v = t[at].reshape(inst, r, G, c)
        if kind in ("forward", "train"):
            mean = v.mean((1, 3), keepdim=True)
            rstd = ((v - mean).pow(2).mean((1, 3), keepdim=True) + EPS).rsqrt()
            stats[which] = torch.stack([mean.reshape(inst, G), rstd.reshape(inst, G)], -1)
            res["y"][at] = act64(((v - mean) * rstd).reshape(inst * r, C) * gamma + beta, False)
        else:
            mean = s["stats"][which][:, :, 0].to(d).reshape(inst, 1, G, 1)
            rstd = s["stats"][which][:, :, 1].to(d).reshape(inst, 1, G, 1)
        k = v if kept is None else kept[at].reshape(inst, r, G, c)
        xn = (k - mean) * rstd
        z = xn.reshape(inst * r, C) * gamma + beta
        if kind in ("restore", "train"):
            res["u"][at] = act64(z, False)
        if kind in ("backward", "train"):
            w = s["dy"][at].to(d) * act64(z, True)
            dbeta += w.sum(0)
            dgamma += (w * xn.reshape(inst * r, C)).sum(0)
            gw = (w * gamma).reshape(inst, r, G, c)
            res["dx"][at] = (rstd * (gw - gw.mean((1, 3), keepdim=True)
                                     - xn * (gw * xn).mean((1, 3), keepdim=True))).reshape(inst * r, C)
            if s["grad_addend"] is not None:
                res["dx"][at] += s["grad_addend"][at].to(d)
    if kind == "restore":
        return {"u": res["u"]}
    if kind in ("forward", "train"):
        out["y"], out["stats"] = res["y"], stats
    if kind == "train":
        out["u"] = res["u"]
    if kind in ("train", "backward"):
        out.update(dx=res["dx"], dgamma=dgamma, dbeta=dbeta)
    return out
