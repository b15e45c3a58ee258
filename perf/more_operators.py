"""Performance cases of what a block of sites that reads other states is made of.

Sites attend to states of another length: the coarse rows of a pooled level to the
fine ones below it, a few latent rows to a whole scene, the points of strokes to the
states of a text, and a stream's newest point to states that stay (``cross_*``).
Around such a block stand its norms: the block's result is normed, gated, added to the
scaled residual, and normed again for the next block, in one pass (``block_*``).
Training clips the gradients of all weights by their global norm (``clip_*``).

``run`` computes the plain form in elementary torch operations in 32 bits (sums of
squares over many tensors in 64), or calls the library's operators where ``own`` is
set.  ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
ALPHA = 0.875  # scale of the residual


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def _named(name, **case):
    return case if name is None else dict(name=name, **case)


def _block(name, rows, channels, dtype, gate=True, train=False):
    """dtype: of the block's rows; "mixed" has them in bf16 beside an fp32 residual."""
    return _named(name, op="block", rows=rows, channels=channels, dtype=dtype, gate=gate,
                  train=train)


def _clip(name, kind, size, dtype, clipped):
    """clipped: the norm is four times its bound, and the results are tensors of their own;
    otherwise it is a quarter of it, and the gradients are clipped in place."""
    return _named(name, op="clip", kind=kind, size=size, dtype=dtype, clipped=clipped)


def _cross(name, samples, queries, keys, heads, kv, dim, dtype, train=False):
    return _named(name, op="cross", samples=samples, queries=queries, keys=keys, heads=heads,
                  kv=kv, dim=dim, dtype=dtype, train=train)


def listed():
    return [
        # one new point of each of 16 strokes: a call that is all latency
        _block("block_points", 16, 64, "bf16"),
        # inference on the fine level of the surface batch, fp32 features, no gate
        _block("block_surfaces", 160003, 96, "f32", gate=False),
        # a training step on wide bf16 rows: forward, every gradient
        _block("block_train", 300001, 256, "bf16", train=True),
        # the same on an odd number of channels, bf16 rows beside an fp32 residual
        _block("block_train_odd", 60007, 75, "mixed", train=True),
        # the gradients of one block of 64 channels
        _clip("clip_block", "block", 64, "f32", True),
        # those of a network of 3x3x3 filters, its channels rising by 32 a layer
        _clip("clip_network", "network", 8, "f32", True),
        # 48 tensors of a large model, fp32 and bf16 in turn, too small to be clipped
        _clip("clip_model", "model", 200000000, "mixed", False),
        # one point of each of 16 strokes against its text
        _cross("cross_points", 16, 16, 4001, 4, 4, 32, "bf16"),
        # one point of each of 128 streams, against 2000 states each
        _cross("cross_streams", 128, 128, 262144, 8, 2, 64, "bf16"),
        # 64 latent rows of each of 4 scenes read all of the scene's sites, fp32
        _cross("cross_latents", 4, 256, 200003, 4, 4, 32, "f32"),
        # training: the coarse rows of 8 scenes read the fine ones
        _cross("cross_train", 8, 16001, 60007, 4, 4, 64, "bf16", train=True),
        # training: the points of 32 pages of strokes read some 40 states of text, fp32
        _cross("cross_train_text", 32, 120011, 1283, 4, 2, 32, "f32", train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(["block", "clip", "cross"], [4, 2, 6])[0]
    train = rng.random() < 0.5
    if op == "block":
        channels = rng.choice([3, 7, 8, 24, 32, 50, 64, 75, 96, 100, 128, 200, 256, 330, 512,
                               1000, 1024, 2048, 4096])
        dtype = rng.choice(["f32", "bf16", "bf16", "mixed"])
        most = 300001 * 256 // {"f32": 2, "bf16": 1, "mixed": 2}[dtype]
        rows = max(1, min(_log(rng, 1, 300001), most // channels))
        return _block(None, rows, channels, dtype, rng.random() < 0.7, train)
    if op == "clip":
        kind = rng.choice(["block", "network", "model"])
        size = {"block": lambda: _log(rng, 8, 512), "network": lambda: rng.randint(1, 12),
                "model": lambda: _log(rng, 1000, 100000000)}[kind]()
        return _clip(None, kind, size, rng.choice(["f32", "bf16", "mixed"]), rng.random() < 0.6)
    kv = rng.choice([1, 1, 2, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 8])
    while heads > 16:
        heads -= kv
    dim = rng.choice([16, 24, 32, 32, 40, 64, 64, 64, 80, 96, 128, 128])
    dtype = "bf16" if rng.random() < 0.6 else "f32"
    narrow = 1 if dtype == "bf16" else 2
    samples = _log(rng, 1, 32)
    queries = _log(rng, 1, 120011)
    if rng.random() < 0.35:  # single rows of streams
        samples = queries = _log(rng, 1, 256)
        train = False
    # (a row that sees one key alone has no gradient of its score)
    keys = max(_log(rng, 1, 262144), 16 * samples if train else 1)
    # no more elements and products than the largest listed cases of the type and direction
    keys = max(1, min(keys, 262144 * 2 * 64 // (kv * dim * narrow)))
    queries = max(1, min(queries, 120011 * 4 * 32 // (heads * dim)))
    wide = heads * max(dim, 32)
    cost = 16001 * 7501 * 4 * 64 // (narrow * (3 if narrow == 2 else 1))
    if not train:
        cost = cost // 2
    while keys > 16 * samples and queries / samples * keys * wide > cost:
        keys = max(16 * samples, keys * 4 // 5)
    while queries > samples and queries / samples * keys * wide > cost:
        queries = max(samples, queries * 4 // 5)
    return _cross(None, samples, queries, keys, heads, kv, dim, dtype, train)


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _types(case):
    """(of the residual, of the block's rows)"""
    if case["dtype"] == "mixed":
        return torch.float32, torch.bfloat16
    return DTYPE[case["dtype"]], DTYPE[case["dtype"]]


def _shapes(case):
    """(shape, type) of each gradient."""
    n, kind = case["size"], case["kind"]
    if kind == "block":  # projections of queries, states, gate and result, and four norms
        shapes = [(n, n), (n, 2 * n), (n, n), (n, n), (n,), (n,), (32,), (32,)]
    elif kind == "network":  # n layers of 3x3x3 filters and the classes
        wide = [1] + [32 * (i + 1) for i in range(n)]
        shapes = [x for a, b in zip(wide, wide[1:]) for x in ((27, a, b), (b,))]
        shapes += [(wide[-1], 101), (101,)]
    else:  # 48 tensors: one of a quarter of all, then ever smaller ones, small odd ones between
        rest, shapes = n, []
        for i in range(24):
            m = max(1, rest // 4 if i < 8 else rest // (24 - i))
            rest = max(0, rest - m)
            shapes += [(m,), (1 + 37 * i,)]
    kinds = {"f32": ["f32"], "bf16": ["bf16"], "mixed": ["f32", "bf16"]}[case["dtype"]]
    return [(s, DTYPE[kinds[i // 2 % len(kinds)]]) for i, s in enumerate(shapes)]


def _lengths(n, b, phase):
    """Rows of each of b samples: uneven, set by the sizes alone; some may be empty."""
    w = [1.0 + 0.5 * math.sin(2.4 * i + phase) for i in range(b)]
    t, cut = sum(w), [0]
    for i in range(b):
        cut.append(cut[-1] + w[i])
    at = [int(round(n * c / t)) for c in cut]
    at[-1] = n
    return [at[i + 1] - at[i] for i in range(b)]


def _both_lengths(case):
    b, q = case["samples"], case["queries"]
    return [1] * b if q == b else _lengths(q, b, 0.7), _lengths(case["keys"], b, 2.9)


def _places(lens):
    """Where each row lies in samples padded to the longest."""
    most = max(lens)
    return torch.cat([i * most + torch.arange(m) for i, m in enumerate(lens)]).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    s = dict(case=case, seed=seed)
    if case["op"] == "block":
        n, c = case["rows"], case["channels"]
        res, typ = _types(case)
        # a residual that several blocks have grown, a block's result of ordinary size
        s["x"], s["f"] = normal(n, c, std=2.0, dtype=res), normal(n, c, std=0.5, dtype=typ)
        s["z"] = normal(n, c, dtype=typ) if case["gate"] else None
        s["wf"], s["wh"] = 1.0 + normal(c, std=0.2), 1.0 + normal(c, std=0.2)
        if case["train"]:
            s["dy"], s["dh"] = normal(n, c, dtype=res), normal(n, c, dtype=typ)
    elif case["op"] == "clip":
        shapes = _shapes(case)
        count = sum(math.prod(t) for t, _ in shapes)
        std = 1e-3  # gradients of a mean over a batch
        s["grads"] = [normal(*t, std=std, dtype=d) for t, d in shapes]
        norm = std * math.sqrt(count)
        s["most"] = norm / 4 if case["clipped"] else norm * 4
        s["out"] = [torch.empty_like(t) for t in s["grads"]] if case["clipped"] else None
    else:
        H, K, D, dt = case["heads"], case["kv"], case["dim"], DTYPE[case["dtype"]]
        ql, kl = _both_lengths(case)
        s["lens"] = ql, kl
        s["places"] = _places(ql), _places(kl)
        s["q_ranges"], s["k_ranges"] = (
            torch.tensor([0] + x, device="cuda").cumsum(0).to(torch.int32) for x in (ql, kl))
        # normalised queries and keys, the queries' learned gains 1.5: scores of N(0, 1.5)
        s["q"] = normal(case["queries"], H, D, std=1.5, dtype=dt)
        s["kv"] = normal(case["keys"], 2 * K * D, dtype=dt)  # one projection of the states
        if case["train"]:
            s["do"] = normal(case["queries"], H, D, dtype=dt)
    return s


def _kv(s):
    c = s["case"]
    x = s["kv"].view(c["keys"], 2 * c["kv"], c["dim"])
    return x[:, :c["kv"]], x[:, c["kv"]:]


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(s):
    return {"block": _run_block, "clip": _run_clip, "cross": _run_cross}[s["case"]["op"]](s)


def _run_block(s):
    c = s["case"]
    x, f, z, wf, wh = s["x"], s["f"], s["z"], s["wf"], s["wh"]
    if own:
        import paper_1505_02890_amd as scn
        y, h = scn.block_norm_fwd(x, f, z, wf, wh, alpha=ALPHA, eps=EPS)
        if not c["train"]:
            return y, h
        d = scn.block_norm_bwd(x, f, z, wf, wh, s["dy"], s["dh"], alpha=ALPHA, eps=EPS)
        grads = [d["dx"], d["df"], d["dwf"], d["dwh"]]
        return (y, h, *grads, d["dz"]) if c["gate"] else (y, h, *grads)
    res, typ = x.dtype, f.dtype
    x, f = x.float(), f.float()
    rf = torch.rsqrt(f.square().mean(1, keepdim=True) + EPS)
    fn = f * rf
    u = fn * wf
    gate = torch.sigmoid(z.float()) if c["gate"] else 1.0
    y = ALPHA * x + gate * u
    ry = torch.rsqrt(y.square().mean(1, keepdim=True) + EPS)
    yn = y * ry
    out = [y.to(res), (yn * wh).to(typ)]
    if c["train"]:
        dh = s["dh"].float()
        dwh = (dh * yn).sum(0)
        a = dh * wh
        dy = s["dy"].float() + ry * (a - yn * (a * yn).mean(1, keepdim=True))
        du = dy * gate
        dwf = (du * fn).sum(0)
        b = du * wf
        df = rf * (b - fn * (b * fn).mean(1, keepdim=True))
        out += [(ALPHA * dy).to(res), df.to(typ), dwf, dwh]
        if c["gate"]:
            out.append((dy * u * gate * (1.0 - gate)).to(typ))
    return tuple(out)


def _run_clip(s):
    grads, most = s["grads"], s["most"]
    if own:
        import paper_1505_02890_amd as scn
        norm = scn.clip_grads(grads, most, out=s["out"])
        return norm, s["out"] or grads
    flat = torch.cat([t.flatten().float() for t in grads]).double()
    norm = flat.square().sum().sqrt()
    scale = torch.clamp(most / norm, max=1.0)
    parts = (flat * scale).split([t.numel() for t in grads])
    return norm.float(), [p.to(t.dtype).view(t.shape) for p, t in zip(parts, grads)]


def _run_cross(s):
    c = s["case"]
    k, v = _kv(s)
    if own:
        import paper_1505_02890_amd as scn
        o, lse = scn.cross_attn_fwd(s["q"], k, v, s["q_ranges"], s["k_ranges"])
        if not c["train"]:
            return o, lse
        d = scn.cross_attn_bwd(s["q"], k, v, o, lse, s["do"], s["q_ranges"], s["k_ranges"])
        return o, lse, d["dq"], d["dk"], d["dv"]
    ql, kl = s["lens"]
    dt = s["q"].dtype
    q, k, v = s["q"].float(), k.float(), v.float()
    do = s["do"].float() if c["train"] else None
    if len(ql) * max(ql) * max(kl) * c["heads"] <= 1 << 28:  # all samples at once, padded
        out = _attend_padded(s, q, k, v, do)
    else:
        out = _attend_samples(s, q, k, v, do)
    return tuple(t if i == 1 else t.to(dt) for i, t in enumerate(out))


def _attend(q, k, v, do, see):
    """q, do [n, K, rows, D], k, v [n, K, keys, D], see [n, 1, 1, keys] or None."""
    scale = 1.0 / math.sqrt(q.shape[-1])
    x = torch.matmul(q, k.transpose(2, 3)) * scale
    if see is not None:
        x = x.masked_fill_(~see, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = (x - top.clamp(min=-3e38)).exp_()
    z = p.sum(-1, keepdim=True)
    p = p / z.clamp(min=1e-30)  # (no key seen: weights of 0)
    o = torch.matmul(p, v)
    lse = top + z.log()
    if do is None:
        return o, lse
    ds = p * (torch.matmul(do, v.transpose(2, 3)) - (do * o).sum(-1, keepdim=True)) * scale
    return (o, lse, torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q),
            torch.matmul(p.transpose(2, 3), do))


def _attend_padded(s, q, k, v, do):
    c = s["case"]
    B, H, K, D = c["samples"], c["heads"], c["kv"], c["dim"]
    G = H // K
    (ql, kl), (qp, kp) = s["lens"], s["places"]
    nq, nk = max(ql), max(kl)

    def rows(t, heads, most, places):  # [rows, heads, D] to [B, K, heads / K * most, D]
        pad = torch.zeros(B * most, heads, D, device="cuda").index_copy_(0, places, t)
        return pad.view(B, most, heads, D).transpose(1, 2).reshape(B, K, -1, D)

    def back(t, heads, most, places):
        return t.reshape(B, heads, most, -1).transpose(1, 2).reshape(B * most, heads, -1)[places]

    kr = s["k_ranges"]
    see = torch.arange(nk, device="cuda")[None] < (kr[1:] - kr[:-1])[:, None]
    r = _attend(rows(q, H, nq, qp), rows(k, K, nk, kp), rows(v, K, nk, kp),
                None if do is None else rows(do, H, nq, qp), see[:, None, None])
    out = [back(r[0], H, nq, qp), back(r[1], H, nq, qp)[..., 0].t().contiguous()]
    if do is not None:
        out += [back(r[2], H, nq, qp), back(r[3], K, nk, kp), back(r[4], K, nk, kp)]
    return out


def _attend_samples(s, q, k, v, do):
    c = s["case"]
    H, K, D = c["heads"], c["kv"], c["dim"]
    G, n = H // K, c["queries"]
    o, lse = torch.zeros(n, H, D, device="cuda"), torch.full((H, n), -math.inf, device="cuda")
    dq, dk, dv = torch.zeros_like(o), torch.zeros_like(k), torch.zeros_like(v)

    def heads(t):  # [rows, heads, D] to [1, K, heads / K * rows, D]
        return t.transpose(0, 1).reshape(1, K, -1, D)

    q0 = k0 = 0
    for m, keys in zip(*s["lens"]):
        kk, vv = k[k0:k0 + keys], v[k0:k0 + keys]
        step = max(64, (1 << 28) // max(1, keys * H))
        for i in range(q0, q0 + m if keys else q0, step):
            r = slice(i, min(i + step, q0 + m))
            w = r.stop - r.start
            a = _attend(heads(q[r]), heads(kk), heads(vv),
                        None if do is None else heads(do[r]), None)
            o[r] = a[0].view(H, w, D).transpose(0, 1)
            lse[:, r] = a[1].view(H, w)
            if do is not None:
                dq[r] = a[2].view(H, w, D).transpose(0, 1)
                dk[k0:k0 + keys] += a[3][0].transpose(0, 1)
                dv[k0:k0 + keys] += a[4][0].transpose(0, 1)
        q0, k0 = q0 + m, k0 + keys
    return [o, lse] if do is None else [o, lse, dq, dk, dv]


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    if case["op"] == "block":
        x, a = case["rows"] * case["channels"], 1 if case["gate"] else 0
        r, t = (torch.finfo(d).bits // 8 for d in _types(case))
        byt, fl = x * (2 * r + (2 + a) * t) + 8 * case["channels"], 16 * x
        if case["train"]:  # dy, dh in; dx, df, dz out
            byt += x * (2 * r + (2 + a) * t) + 8 * case["channels"]
            fl += 32 * x
        return dict(bytes=byt, flops=fl)
    if case["op"] == "clip":
        shapes = _shapes(case)
        byt = sum(math.prod(t) * torch.finfo(d).bits // 8 for t, d in shapes)
        count = sum(math.prod(t) for t, _ in shapes)
        return dict(bytes=byt * (2 if case["clipped"] else 1) + 4, flops=2 * count)
    H, K, D, q, k = (case[n] for n in ("heads", "kv", "dim", "queries", "keys"))
    e = 2 if case["dtype"] == "bf16" else 4
    pairs = sum(a * b for a, b in zip(*_both_lengths(case)))
    byt = (2 * q * H + 2 * k * K) * D * e + 4 * H * q
    fl = 4 * D * H * pairs
    if case["train"]:
        byt += (2 * q * H + 2 * k * K) * D * e  # do in; dq, dk, dv out
        fl += 10 * D * H * pairs
    return dict(bytes=byt, flops=fl)


# --------------------------------------------------------------------------
# the definition, in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"block": _exact_block, "clip": _exact_clip, "cross": _exact_cross}[case["op"]](s)


def _unit(t):
    """(rows of mean square 1 but for EPS, what they were divided by)"""
    size = ((t ** 2).sum(1, keepdim=True) / t.shape[1] + EPS) ** 0.5
    return t / size, size


def _unit_grad(unit, size, g):
    return (g - unit * ((unit * g).sum(1, keepdim=True) / g.shape[1])) / size


def _exact_block(s):
    c = s["case"]
    wf, wh = s["wf"].double(), s["wh"].double()
    f, fs = _unit(s["f"].double())
    part = f * wf
    if c["gate"]:
        e = torch.exp(-s["z"].double())
        y = s["x"].double() * ALPHA + part / (1 + e)
    else:
        y = s["x"].double() * ALPHA + part
    h, hs = _unit(y)
    out = [y, h * wh]
    if c["train"]:
        dh = s["dh"].double()
        dy = _unit_grad(h, hs, dh * wh) + s["dy"].double()
        dpart = dy / (1 + e) if c["gate"] else dy
        out += [dy * ALPHA, _unit_grad(f, fs, dpart * wf), (dpart * f).sum(0), (dh * h).sum(0)]
        if c["gate"]:
            out.append(dy * part * e / (1 + e) ** 2)
    return tuple(out)


def _exact_clip(s):
    total = math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in s["grads"]))
    by = s["most"] / total if total > s["most"] else 1.0
    return torch.tensor(total, dtype=torch.float64), [t.double() * by for t in s["grads"]]


def _exact_cross(s):
    c = s["case"]
    H, K, D, n = c["heads"], c["kv"], c["dim"], c["queries"]
    k, v = _kv(s)
    f64 = dict(dtype=torch.float64, device="cuda")
    o, lse = torch.zeros(n, H, D, **f64), torch.full((H, n), -math.inf, **f64)
    dq, dk, dv = torch.zeros(n, H, D, **f64), torch.zeros(k.shape, **f64), torch.zeros(k.shape, **f64)
    q0 = k0 = 0
    for m, keys in zip(*s["lens"]):
        ks = slice(k0, k0 + keys)
        k0 += keys
        q1 = q0 + m
        for i in range(q0, q1 if keys else q0, 4096):
            r = slice(i, min(i + 4096, q1))
            for h in range(H):
                j = h * K // H
                kd, vd, qd = k[ks, j].double(), v[ks, j].double(), s["q"][r, h].double()
                w = qd @ kd.T
                w /= D ** 0.5
                lse[h, r] = torch.logsumexp(w, 1)
                w -= lse[h, r][:, None]
                w.exp_()
                o[r, h] = w @ vd
                if c["train"]:
                    g = s["do"][r, h].double()
                    dv[ks, j] += w.T @ g
                    dw = g @ vd.T
                    dw -= (g * o[r, h]).sum(1, keepdim=True)
                    dw *= w
                    dw /= D ** 0.5
                    dq[r, h] = dw @ kd
                    dk[ks, j] += dw.T @ qd
        q0 = q1
    return (o, lse, dq, dk, dv) if c["train"] else (o, lse)
