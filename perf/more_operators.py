"""Cases of the attention operators: what a program does that lets every node of a
sub-graph see every other one, beside message passing within a radius.

Queries and keys are normed for each head and rotated by the nodes' coordinates;
then every query attends to the keys of its own packed sub-graph, with scores that
a tanh may cap and that fall with the distance of the two nodes.  Training takes
the gradients; a field is read out at a few probe points with few queries over
many keys.

Sizes are those of the repository's workloads and their neighbours: one row, about a
thousand nodes (a sampled square), packed sub-domains, 262,144 nodes (a channel
slab); latent widths of 64 to 512 in heads of 16 to 128.
"""

import math

import torch

own = False

EPS = 1e-6
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def rotate(name, kind, n, H, Hk, hd, type, rot, axes, layout, norm=True):
    return dict(name=name, kind=kind, n=n, H=H, Hk=Hk, hd=hd, type=type, rot=rot, axes=axes, layout=layout, norm=norm)


def attend(name, kind, nq, nk, segs, H, Hk, hd, type, dim, cap):
    return dict(name=name, kind=kind, nq=nq, nk=nk, segs=segs, H=H, Hk=Hk, hd=hd, type=type, dim=dim, cap=cap)


def listed():
    return [
        # one probe point's query and key: the smallest call (latency)
        rotate("rotate-1", "rotate", 1, 8, 2, 64, "bf16", 64, 2, "half"),
        # all nodes of a channel slab, three coordinates, the last part of each head left unrotated
        rotate("rotate-262k", "rotate", 262144, 8, 8, 64, "bf16", 48, 3, "half"),
        # training step on a small square, float32
        rotate("rotate-grad-1k", "rotate-grad", 1000, 4, 4, 32, "f32", 32, 2, "interleaved"),
        # training step on packed sub-domains, an odd number of nodes, shared key heads
        rotate("rotate-grad-100k", "rotate-grad", 99991, 8, 2, 64, "bf16", 64, 2, "interleaved"),
        # evaluation of a small sampled square in float32
        attend("attend-1k", "attend", 1024, 1024, 1, 4, 4, 32, "f32", 2, 0.0),
        # evaluation of 37 sub-domains of one domain packed one after another, an odd number of nodes
        attend("attend-packed-33k", "attend", 32749, 32749, 37, 4, 4, 32, "bf16", 2, 0.0),
        # evaluation of one large sub-graph, wide heads, shared key heads, capped scores
        attend("attend-16k", "attend", 16384, 16384, 1, 8, 2, 128, "bf16", 0, 50.0),
        # a field read out at five probe points of a channel slab
        attend("probe-262k", "attend", 5, 262144, 1, 8, 2, 64, "bf16", 3, 0.0),
        # one probe point in each of 37 packed sub-domains
        attend("probe-packed-100k", "attend", 37, 99991, 37, 8, 8, 64, "bf16", 0, 0.0),
        # training step on a small square, float32
        attend("train-1k", "train", 1000, 1000, 1, 4, 4, 32, "f32", 2, 30.0),
        # training step on sixteen packed sub-domains of a channel, distance bias, shared key heads
        attend("train-packed-33k", "train", 32768, 32768, 16, 8, 4, 64, "bf16", 3, 0.0),
        # the largest: training step on one large sub-graph
        attend("train-16k", "train", 16384, 16384, 1, 16, 16, 64, "bf16", 0, 0.0),
    ]


def spread(rng, low, high):
    """A whole number of [low, high], spread over its logarithm."""
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate-grad", "attend", "attend", "probe", "train", "train"])
    H = rng.choice([1, 2, 3, 4, 6, 8, 16])
    Hk = rng.choice([g for g in range(1, H + 1) if H % g == 0])
    hd = rng.choice([32, 64, 128, 8 * rng.randrange(1, 17)])
    type = rng.choice(["f32", "bf16", "bf16"])
    if kind.startswith("rotate"):
        axes = rng.choice([a for a in (1, 2, 3) if 2 * a <= hd])
        rot = 2 * axes * rng.randrange(1, hd // (2 * axes) + 1)
        n = spread(rng, 1, min(262144, 262144 * 16 * 64 // ((H + Hk) * hd) // (2 if type == "f32" or kind == "rotate-grad" else 1)))
        return rotate("", kind, n, H, Hk, hd, type, rot, axes, rng.choice(["half", "interleaved"]), rng.random() < 0.8)
    dim = rng.choice([0, 1, 2, 3])
    cap = rng.choice([0.0, 0.0, round(rng.uniform(5.0, 60.0), 1)])
    if kind == "probe":
        segs = rng.choice([1, spread(rng, 2, 64)])
        nq = max(segs, spread(rng, 1, 128))
        nk = spread(rng, 64 * segs, 262144 // (2 if type == "f32" else 1))
        return attend("", "attend", nq, nk, segs, H, Hk, hd, type, dim, cap)
    # the products of all pairs are at most a quarter of the largest listed case's, float32 ones 32 times fewer, and a pass
    # over padded segments holds at most 2^31 scores
    segs = rng.choice([1, 1, spread(rng, 2, 48)])
    pairs = 16384 ** 2 * 16 * 64 // (4 if type == "bf16" else 128)
    most = int(min(32768, (pairs * segs / (H * hd)) ** 0.5, (2 ** 31 * segs / (8 * H)) ** 0.5))
    nq = spread(rng, 4 * segs, most)
    nk = nq if rng.random() < 0.7 else spread(rng, 4 * segs, most)
    return attend("", kind, nq, nk, segs, H, Hk, hd, type, dim, cap)


def bounds(n, segs):
    """Where the packed segments begin and end: of unequal lengths, a row at least in each."""
    w = [0.25 + ((i * 0.6180339887) % 1.0) * 2.0 for i in range(segs)]
    total, at, ends = sum(w), 0.0, [0]
    for i, v in enumerate(w):
        at += v
        ends.append(max(ends[-1] + 1, min(n - (segs - 1 - i), int(round(n * at / total)))))
    ends[-1] = n
    return ends


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    H, Hk, hd, kind = case["H"], case["Hk"], case["hd"], case["kind"]
    dt = DTYPES[case["type"]]
    f32 = dict(device=dev, dtype=torch.float32)

    def normal(*shape):
        return torch.randn(*shape, generator=g, **f32)

    s = dict(case=case)
    if kind in ("rotate", "rotate-grad"):
        n, pairs = case["n"], case["rot"] // 2
        # a projection's outputs: channels with scales of their own
        s["q"] = (normal(n, H * hd) * torch.exp(0.4 * normal(H * hd))).to(dt)
        s["k"] = (normal(n, Hk * hd) * torch.exp(0.4 * normal(Hk * hd))).to(dt)
        s["gq"] = 1.0 + 0.2 * normal(hd) if case["norm"] else None
        s["gk"] = 1.0 + 0.2 * normal(hd) if case["norm"] else None
        # coordinates in units of the sampling distance, frequencies from one to a thousandth of that
        s["pos"] = 600.0 * torch.rand(n, case["axes"], generator=g, **f32)
        per = pairs // case["axes"]
        s["freq"] = torch.exp(torch.arange(per, **f32) * (-math.log(1000.0) / per)).repeat(case["axes"])
        names = [("q", H), ("k", Hk)]
        if kind == "rotate-grad":
            s["dyq"], s["dyk"] = normal(n, H * hd).to(dt), normal(n, Hk * hd).to(dt)
            if case["norm"]:
                s["dgq"], s["dgk"] = torch.empty(hd, **f32), torch.empty(hd, **f32)
        for name, heads in names:
            s[name + "_out"] = torch.empty(n, heads * hd, device=dev, dtype=dt)
        return s
    nq, nk, segs = case["nq"], case["nk"], case["segs"]
    s["q"], s["k"], s["v"] = normal(nq, H * hd).to(dt), normal(nk, Hk * hd).to(dt), normal(nk, Hk * hd).to(dt)
    s["q_ends"], s["k_ends"] = bounds(nq, segs), bounds(nk, segs)
    s["q_seg"] = torch.tensor(s["q_ends"], dtype=torch.int32, device=dev)
    s["k_seg"] = s["q_seg"] if nq == nk else torch.tensor(s["k_ends"], dtype=torch.int32, device=dev)
    s["pos"] = s["k_pos"] = s["slopes"] = None
    if case["dim"]:
        s["pos"] = torch.rand(nq, case["dim"], generator=g, **f32)
        s["k_pos"] = s["pos"] if nq == nk else torch.rand(nk, case["dim"], generator=g, **f32)
        # slopes of the heads: from 8 for a domain's length downwards
        s["slopes"] = 8.0 * torch.exp2(torch.arange(H, **f32) * (-8.0 / H))
    s["out"] = torch.empty(nq, H * hd, device=dev, dtype=dt)
    s["lse"] = torch.empty(nq, H, **f32)
    if kind == "train":
        s["dout"] = normal(nq, H * hd).to(dt)
        s["dq"] = torch.empty(nq, H * hd, device=dev, dtype=dt)
        s["dk"], s["dv"] = (torch.empty(nk, Hk * hd, device=dev, dtype=dt) for _ in range(2))
    return s


# ---------------------------------------------------------------- plain form

def turned(u, pos, freq, rot, axes, layout, back):
    """Rows [n, heads, hd] with their pairs rotated by the coordinates' angles (back: the other way)."""
    pairs = rot // 2
    at = pos.double().repeat_interleave(pairs // axes, 1) * freq.double()
    c, s = torch.cos(at).float()[:, None], torch.sin(at).float()[:, None]
    s = -s if back else s
    r = u[:, :, :rot]
    if layout == "half":
        a, b = r[:, :, :pairs], r[:, :, pairs:]
        r = torch.cat([a * c - b * s, a * s + b * c], 2)
    else:
        a, b = r[:, :, 0::2], r[:, :, 1::2]
        r = torch.stack([a * c - b * s, a * s + b * c], 3).flatten(2)
    return torch.cat([r, u[:, :, rot:]], 2)


def plain_rotate(s, x, gamma, heads):
    case = s["case"]
    u = x.float().view(case["n"], heads, case["hd"])
    if gamma is not None:
        u = u / torch.sqrt((u * u).mean(2, keepdim=True) + EPS) * gamma
    return turned(u, s["pos"], s["freq"], case["rot"], case["axes"], case["layout"], False).flatten(1).to(x.dtype)


def plain_rotate_grad(s, x, dy, gamma, heads):
    case = s["case"]
    u = x.float().view(case["n"], heads, case["hd"])
    g = turned(dy.float().view_as(u), s["pos"], s["freq"], case["rot"], case["axes"], case["layout"], True)
    if gamma is None:
        return g.flatten(1).to(x.dtype), None
    r = 1.0 / torch.sqrt((u * u).mean(2, keepdim=True) + EPS)
    xn, w = u * r, g * gamma
    dx = r * (w - xn * (w * xn).mean(2, keepdim=True))
    return dx.flatten(1).to(x.dtype), (g * xn).sum((0, 1))


def padded(ends, dev):
    """Rows [segments, longest] of packed segments, side by side, and which of them there are."""
    e = torch.tensor(ends, device=dev)
    longest = max(b - a for a, b in zip(ends, ends[1:]))
    row = e[:-1, None] + torch.arange(longest, device=dev)
    there = row < e[1:, None]
    return torch.where(there, row, torch.zeros_like(row)), there


def plain_attend(s):
    """All segments at once, padded to the longest: scores [segments, heads, queries, keys]."""
    case = s["case"]
    H, Hk, hd, cap, dev = case["H"], case["Hk"], case["hd"], case["cap"], s["q"].device
    qi, q_there = padded(s["q_ends"], dev)
    ki, k_there = padded(s["k_ends"], dev)
    scale = hd ** -0.5
    S, Lq, Lk = len(s["q_ends"]) - 1, qi.shape[1], ki.shape[1]

    def rows(t, heads, index):
        """[segments, key heads, query heads to each, rows, hd]"""
        return t.float()[index].view(S, index.shape[1], Hk, heads // Hk, hd).permute(0, 2, 3, 1, 4)

    q, k, v = rows(s["q"], H, qi), rows(s["k"], Hk, ki), rows(s["v"], Hk, ki)
    q = q.reshape(S, Hk, H // Hk * Lq, hd)
    k, v = k.reshape(S, Hk, Lk, hd), v.reshape(S, Hk, Lk, hd)
    b = (q @ k.transpose(2, 3)).mul_(scale)
    fall = None
    if cap:
        b = b.div_(cap).tanh_()
        fall = 1.0 - b * b if case["kind"] == "train" else None
        b = b.mul_(cap)
    b = b.view(S, Hk, H // Hk, Lq, Lk)
    if case["dim"]:
        d = s["pos"][qi][:, :, None] - s["k_pos"][ki][:, None]
        d = (d * d).sum(3).sqrt()
        b = b.sub_(s["slopes"].view(Hk, H // Hk, 1, 1) * d[:, None, None])
    b = b.masked_fill_(~k_there[:, None, None, None], -math.inf)
    top = b.amax(4, keepdim=True)
    P = b.sub_(top).exp_()
    total = P.sum(4, keepdim=True)
    P = P.div_(total).view(S, Hk, H // Hk * Lq, Lk)

    def back(t, heads, there):
        """Packed rows [n, heads hd] again."""
        return t.view(S, Hk, heads // Hk, -1, hd).permute(0, 3, 1, 2, 4).reshape(S, -1, heads * hd)[there].to(s["q"].dtype)

    o = P @ v
    lse = (top + total.log()).view(S, H, Lq).transpose(1, 2)[q_there]
    out = {"out": back(o, H, q_there), "lse": lse}
    if case["kind"] == "train":
        do = rows(s["dout"], H, qi) * q_there[:, None, None, :, None]
        do = do.reshape(S, Hk, H // Hk * Lq, hd)
        out["dv"] = back(P.transpose(2, 3) @ do, Hk, k_there)
        dS = (do @ v.transpose(2, 3)).sub_((do * o).sum(3, keepdim=True)).mul_(P)
        if fall is not None:
            dS = dS.mul_(fall)
        out["dq"] = back((dS @ k).mul_(scale), H, q_there)
        out["dk"] = back((dS.transpose(2, 3) @ q).mul_(scale), Hk, k_there)
    return out


def plain(s):
    case = s["case"]
    if case["kind"] == "rotate":
        return {"q": plain_rotate(s, s["q"], s["gq"], case["H"]), "k": plain_rotate(s, s["k"], s["gk"], case["Hk"])}
    if case["kind"] == "rotate-grad":
        dq, dgq = plain_rotate_grad(s, s["q"], s["dyq"], s["gq"], case["H"])
        dk, dgk = plain_rotate_grad(s, s["k"], s["dyk"], s["gk"], case["Hk"])
        return {"dq": dq, "dk": dk, **({"dgq": dgq, "dgk": dgk} if case["norm"] else {})}
    return plain_attend(s)


# ------------------------------------------------------------ the framework's

_handle = []


def kernels(s):
    import paper_2402_15106_amd as dm
    if not _handle:
        _handle.append(dm.Dsmp(0))
    lib, case = _handle[0], s["case"]
    H, Hk, hd = case["H"], case["Hk"], case["hd"]
    dtype = {"f32": dm.F32, "bf16": dm.BF16}[case["type"]]
    if case["kind"] in ("rotate", "rotate-grad"):
        layout = {"half": dm.ROTATE_HALF, "interleaved": dm.ROTATE_INTERLEAVED}[case["layout"]]
        desc = dm.rotate_desc(H, Hk, hd, dtype, case["rot"], axes=case["axes"], layout=layout, norm=case["norm"], eps=EPS)
        if case["kind"] == "rotate":
            q, k = lib.dsmp_qk_rotate_forward(desc, s["q"], s["k"], s["gq"], s["gk"], s["pos"], s["freq"],
                                              q_out=s["q_out"], k_out=s["k_out"])
            return {"q": q, "k": k}
        grads = {"dgamma_q": s["dgq"], "dgamma_k": s["dgk"]} if case["norm"] else None
        dq, dk, _ = lib.dsmp_qk_rotate_backward(desc, s["q"], s["k"], s["gq"], s["gk"], s["pos"], s["freq"], s["dyq"],
                                                s["dyk"], grad_q=s["q_out"], grad_k=s["k_out"], grads=grads)
        return {"dq": dq, "dk": dk, **({"dgq": s["dgq"], "dgk": s["dgk"]} if case["norm"] else {})}
    desc = dm.attention_desc(H, Hk, hd, dtype, dim=case["dim"], cap=case["cap"])
    at = dict(segments=s["q_seg"], k_segments=s["k_seg"], pos=s["pos"], k_pos=s["k_pos"], slopes=s["slopes"])
    out, lse = lib.dsmp_attention_forward(desc, s["q"], s["k"], s["v"], out=s["out"], lse=s["lse"], **at)
    res = {"out": out, "lse": lse}
    if case["kind"] == "train":
        res["dq"], res["dk"], res["dv"] = lib.dsmp_attention_backward(
            desc, s["q"], s["k"], s["v"], out, lse, s["dout"], grad_q=s["dq"], grad_k=s["dk"], grad_v=s["dv"], **at)
    return res


def run(state):
    return kernels(state) if own else plain(state)


def work(case):
    H, Hk, hd, kind = case["H"], case["Hk"], case["hd"], case["kind"]
    e = {"f32": 4, "bf16": 2}[case["type"]]
    if kind in ("rotate", "rotate-grad"):
        n, el = case["n"], case["n"] * (H + Hk) * hd
        tables = 4 * n * case["axes"] + 2 * case["rot"] + (8 * hd if case["norm"] else 0)
        if kind == "rotate":
            return {"bytes": 2 * el * e + tables, "flops": 7 * el}
        return {"bytes": 3 * el * e + tables + (8 * hd if case["norm"] else 0), "flops": 14 * el}
    nq, nk = case["nq"], case["nk"]
    a, b = bounds(nq, case["segs"]), bounds(nk, case["segs"])
    pairs = H * sum((a[i + 1] - a[i]) * (b[i + 1] - b[i]) for i in range(case["segs"]))
    places = 4 * case["dim"] * (nq + nk)
    data = (2 * nq * H + 2 * nk * Hk) * hd * e + 4 * nq * H + places
    if kind == "attend":
        return {"bytes": data, "flops": pairs * 4 * hd}
    # the gradients' pass reads q, k, v, out, lse and the gradient of out, and writes three gradients
    return {"bytes": data + (4 * nq * H + 4 * nk * Hk) * hd * e + 4 * nq * H + places, "flops": pairs * 14 * hd}


# ------------------------------------------------------------ 64 bits

def exact_rotate(case, s):
    d = torch.float64
    n, hd, rot, axes = case["n"], case["hd"], case["rot"], case["axes"]
    half = rot // 2
    angle = torch.empty(n, half, dtype=d, device=s["q"].device)
    for p in range(half):
        angle[:, p] = s["pos"][:, p * axes // half].to(d) * s["freq"][p].to(d)
    first = torch.arange(half, device=angle.device)
    first, second = (first, first + half) if case["layout"] == "half" else (2 * first, 2 * first + 1)
    z = torch.polar(torch.ones_like(angle), angle)[:, None]
    out = {}
    for name, heads in (("q", case["H"]), ("k", case["Hk"])):
        x = s[name].to(d).view(n, heads, hd)
        gamma = s["g" + name].to(d) if case["norm"] else torch.ones(hd, dtype=d, device=x.device)
        inv = (x.pow(2).mean(2, keepdim=True) + EPS).rsqrt() if case["norm"] else torch.ones_like(x[:, :, :1])
        if case["kind"] == "rotate":
            y = x * inv * gamma
            w = torch.complex(y[:, :, first], y[:, :, second]) * z
            y[:, :, first], y[:, :, second] = w.real, w.imag
            out[name] = y.reshape(n, heads * hd)
            continue
        g = s["dy" + name].to(d).view(n, heads, hd).clone()
        w = torch.complex(g[:, :, first], g[:, :, second]) * z.conj()
        g[:, :, first], g[:, :, second] = w.real, w.imag
        dx = g * gamma
        if case["norm"]:
            dx = inv * (dx - x * inv * inv * (dx * x).mean(2, keepdim=True))
            out["dg" + name] = (g * x * inv).sum((0, 1))
        out["d" + name] = dx.reshape(n, heads * hd)
    return out


def exact(case, seed):
    """The same from the definitions in 64 bits, one segment and head at a time."""
    s = prepare(case, seed)
    if case["kind"] in ("rotate", "rotate-grad"):
        return exact_rotate(case, s)
    d = torch.float64
    H, Hk, hd, cap, train = case["H"], case["Hk"], case["hd"], case["cap"], case["kind"] == "train"
    q, k, v = (s[x].to(d).view(s[x].shape[0], -1, hd) for x in "qkv")
    o, lse = torch.zeros_like(q), torch.zeros(case["nq"], H, dtype=d, device=q.device)
    if train:
        do = s["dout"].to(d).view_as(q)
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for i in range(case["segs"]):
        a, b = slice(s["q_ends"][i], s["q_ends"][i + 1]), slice(s["k_ends"][i], s["k_ends"][i + 1])
        far = torch.cdist(s["pos"][a].to(d), s["k_pos"][b].to(d), compute_mode="donot_use_mm_for_euclid_dist") if case["dim"] else None
        for h in range(H):
            j = h // (H // Hk)
            x = torch.mm(q[a, h], k[b, j].t().contiguous()) / math.sqrt(hd)
            t = torch.tanh(x / cap) if cap else None
            x = cap * t if cap else x
            if far is not None:
                x = x - float(s["slopes"][h]) * far
            lse[a, h] = torch.logsumexp(x, 1)
            x = torch.exp(x - lse[a, h][:, None])
            o[a, h] = torch.mm(x, v[b, j].contiguous())
            if train:
                e = do[a, h].contiguous()
                dv[b, j] += torch.mm(x.t(), e)
                x = x * (torch.mm(e, v[b, j].t().contiguous()) - (e * o[a, h]).sum(1, keepdim=True)) / math.sqrt(hd)
                x = x * (1.0 - t * t) if cap else x
                dq[a, h] = torch.mm(x, k[b, j].contiguous())
                dk[b, j] += torch.mm(x.t(), q[a, h].contiguous())
    out = {"out": o.flatten(1), "lse": lse}
    if train:
        out.update(dq=dq.flatten(1), dk=dk.flatten(1), dv=dv.flatten(1))
    return out
