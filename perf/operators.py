"""Performance cases of attention among the active sites.

A program that lets the sites of a sample see each other beyond a filter's reach
takes the queries, keys and values of every active site (one projection, side by
side in one matrix), normalises each head's queries and keys and rotates them by
the site's lattice coordinates (``rotate_*``), and attends within each sample,
whose rows lie together in key order: among all its sites, among the nearest in
that order, or causally along a stroke, with the first sites always visible
(``attend_*``).  A program that receives strokes point by point attends from each
stream's newest point over a cache of its last points and its first ones
(``step_*``).

``run`` computes the plain form in elementary torch operations in 32 bits, or
calls the library's operators where ``own`` is set.  ``exact`` is the definition
in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
BASE = 100.0  # a turn of the slowest pair spans a few hundred sites, the grids' extent


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def _named(name, **case):
    return case if name is None else dict(name=name, **case)


def _rotate(name, rows, heads, kv, dim, dtype, ndim=3, extent=128, train=False):
    return _named(name, op="rotate", rows=rows, heads=heads, kv=kv, dim=dim, dtype=dtype,
                  ndim=ndim, extent=extent, train=train)


def _attend(name, samples, rows, heads, kv, dim, dtype, left=-1, right=-1, sinks=0, train=False):
    return _named(name, op="attend", samples=samples, rows=rows, heads=heads, kv=kv,
                  dim=dim, dtype=dtype, left=left, right=right, sinks=sinks, train=train)


def _step(name, streams, capacity, heads, kv, dim, dtype, left=-1, sinks=0, full=False):
    return _named(name, op="step", streams=streams, capacity=capacity, heads=heads,
                  kv=kv, dim=dim, dtype=dtype, left=left, sinks=sinks, full=full)


def listed():
    return [
        # one new point of each of 16 strokes: a call that is all latency
        _rotate("rotate_points", 16, 4, 4, 32, "bf16", extent=64),
        # inference on the coarse levels of the surface batch, fp32 features
        _rotate("rotate_f32", 131072, 8, 2, 32, "f32"),
        # a training step's calls on the surface batch: forward, and the gradients of both
        # inputs and both weights
        _rotate("rotate_train", 300001, 4, 4, 64, "bf16", train=True),
        # one knotted stroke of 400 sites, each attending to those before it
        _attend("attend_stroke", 1, 400, 2, 2, 32, "f32", right=0),
        # 16 curves of 1000 to 3000 steps, causal, four query heads on one of keys
        _attend("attend_curves", 16, 32001, 4, 1, 64, "bf16", right=0),
        # inference on 32 surfaces, windows of 257 sites in key order and four sinks
        _attend("attend_surfaces", 32, 160003, 8, 2, 32, "bf16", 128, 128, 4),
        # one large scene, every site sees every other, wide heads
        _attend("attend_scene", 1, 16384, 2, 2, 128, "bf16"),
        # training on 8 scenes, wide windows: forward and every gradient
        _attend("attend_train", 8, 60007, 4, 4, 64, "bf16", 512, 512, 1, train=True),
        # the same on fp32 features, 16 curves, causal windows
        _attend("attend_train_f32", 16, 34567, 4, 2, 32, "f32", 255, 0, 2, train=True),
        # one point of each of 16 strokes against its last 257 points and first four
        _step("step_strokes", 16, 300, 4, 4, 32, "bf16", 256, 4),
        # 128 streams, rings of 2048 points
        _step("step_streams", 128, 2064, 8, 2, 64, "bf16", 2047, 16),
        # one stream that sees all of its 262143 points, fp32
        _step("step_long", 1, 262144, 4, 4, 32, "f32", full=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    # query heads on as many heads of keys or on fewer, widths that fill a tile or do not
    kv = rng.choice([1, 1, 2, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 8])
    while heads > 16:
        heads -= kv
    return heads, kv, rng.choice([16, 24, 32, 32, 40, 64, 64, 64, 80, 96, 128, 128])


def draw(rng):
    op = rng.choices(["rotate", "attend", "step"], [3, 6, 3])[0]
    heads, kv, dim = _heads(rng)
    dtype = "bf16" if rng.random() < 0.6 else "f32"
    train = rng.random() < 0.5
    if op == "rotate":
        ndim = rng.randint(1, 4)
        most = 300001 * 8 * 64 * (1 if dtype == "bf16" else 0.5)  # the largest case's channels
        rows = min(_log(rng, 1, 300001), int(most / ((heads + kv) * dim)))
        return _rotate(None, rows, heads, kv, dim, dtype, ndim, rng.choice([32, 64, 128, 512]),
                       train)
    if op == "step":
        sinks = rng.choice([0, 0, 1, 4, 16, 63])
        capacity = sinks + _log(rng, 1, 262144)
        row = kv * dim * (2 if dtype == "bf16" else 4)
        streams = max(1, min(_log(rng, 1, 256), int(128 * 2064 * 256 / (capacity * row))))
        capacity = min(capacity, max(sinks + 1, 128 * 2064 * 256 // row))
        ring = capacity - sinks
        left = -1 if rng.random() < 0.4 else rng.randint(0, ring - 1)
        return _step(None, streams, capacity, heads, kv, dim, dtype, left, sinks,
                     rng.random() < 0.3)
    rows = _log(rng, 1, 160003)
    samples = rng.randint(1, 32)
    kind = rng.choice(["all", "causal", "window", "window", "causal window"])
    left = right = -1
    if kind.endswith("window"):
        left = _log(rng, 1, 1025) - 1
        right = left if kind == "window" else 0
    elif kind == "causal":
        right = 0
    sinks = rng.choice([0, 0, 1, 4, 17]) if left >= 0 else 0
    # no more pairs and channels than the largest listed case of its type
    cost = {("bf16", False): 160003 * 261 * 8 * 32, ("bf16", True): 60007 * 1026 * 4 * 64,
            ("f32", False): 34567 * 258 * 4 * 32 * 3, ("f32", True): 34567 * 258 * 4 * 32}
    cost = cost[dtype, train]
    most = {False: 160003 * 20 * 32, True: 60007 * 16 * 64}[train]  # ... nor more feature elements
    wide = heads * max(dim, 32)
    rows = max(1, min(rows, most // (2 * (heads + kv) * dim * (2 if dtype == "f32" else 1))))
    while rows > 1 and rows * wide * max(256, _reach(rows, samples, left, right, sinks)) > cost:
        rows = max(1, int(rows * 0.8))
    return _attend(None, samples, rows, heads, kv, dim, dtype, left, right, sinks, train)


def _reach(rows, samples, left, right, sinks):
    # sites that a site sees, about
    n = rows / samples * 1.3 + 1
    lo = n / 2 if left < 0 else min(left, n)
    hi = n / 2 if right < 0 else min(right, n)
    return lo + hi + 1 + sinks


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _sections(dim, ndim):
    """Channel pairs of each axis: even shares, the first axes one more."""
    p = dim // 2
    return [p // ndim + (1 if a < p % ndim else 0) for a in range(ndim)]


def _lengths(case):
    """Sites of each sample: uneven, set by the sizes alone; some samples may be empty."""
    n, b = case["rows"], case["samples"]
    w = [1.0 + 0.5 * math.sin(2.4 * i + 0.7) for i in range(b)]
    t, cut = sum(w), [0]
    for i in range(b):
        cut.append(cut[-1] + w[i])
    at = [int(round(n * c / t)) for c in cut]
    at[-1] = n
    return [at[i + 1] - at[i] for i in range(b)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    H, K, D = case["heads"], case["kv"], case["dim"]
    dt = DTYPE[case["dtype"]]

    def normal(*shape, std=1.0, dtype=None):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype or dt)

    s = dict(case=case, seed=seed)
    if case["op"] == "rotate":
        n, nd = case["rows"], case["ndim"]
        s["qkv"] = normal(n, (H + 2 * K) * D)
        s["wq"], s["wk"] = (1.0 + 0.2 * normal(D, dtype=torch.float32) for _ in range(2))
        xs = torch.randint(0, case["extent"], (n, nd), generator=g, device="cuda")
        b = torch.sort(torch.randint(0, 8, (n, 1), generator=g, device="cuda"), dim=0).values
        s["coords"] = torch.cat([b, xs], 1).to(torch.int32).contiguous()
        sec = _sections(D, nd)
        s["sections"] = sec
        s["freq"] = torch.cat([BASE ** (-torch.arange(m, device="cuda", dtype=torch.float32) / m)
                               for m in sec if m])
        if case["train"]:
            s["dq"], s["dk"] = normal(n, H, D), normal(n, K, D)
    elif case["op"] == "attend":
        n = case["rows"]
        lens = _lengths(case)
        s["lens"] = lens
        s["ranges"] = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
        # normalised queries and keys, the queries' learned gains 1.5: scores of N(0, 1.5)
        qkv = normal(n, H + 2 * K, D, dtype=torch.float32)
        qkv[:, :H] *= 1.5
        s["qkv"] = qkv.to(dt).view(n, (H + 2 * K) * D)
        if case["train"]:
            s["do"] = normal(n, H, D)
    else:
        B, C = case["streams"], case["capacity"]
        s["new"] = normal(B, (H + 2 * K) * D)
        s["k_cache"], s["v_cache"] = normal(B, C, K, D), normal(B, C, K, D)
        # from streams that just began to rings that went round
        if case["full"]:
            length = torch.full((B,), C - 1, device="cuda")
        else:
            length = torch.randint(0, 3 * C, (B,), generator=g, device="cuda")
        s["length"] = length.to(torch.int32)
    return s


def _parts(x, H, K, D):
    x = x.view(x.shape[0], H + 2 * K, D)
    return x[:, :H], x[:, H:H + K], x[:, H + K:]


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(s):
    return {"rotate": _run_rotate, "attend": _run_attend, "step": _run_step}[s["case"]["op"]](s)


def _bound(v):
    return None if v < 0 else v


def _run_rotate(s):
    c = s["case"]
    q, k, _ = _parts(s["qkv"], c["heads"], c["kv"], c["dim"])
    if own:
        import paper_1505_02890_amd as scn
        plan = (s["wq"], s["wk"], s["coords"], s["freq"], s["sections"])
        qr, kr = scn.norm_rotate_fwd(q, k, *plan, eps=EPS)
        if not c["train"]:
            return qr, kr
        d = scn.norm_rotate_bwd(q, k, *plan, s["dq"], s["dk"], eps=EPS)
        return qr, kr, d["dq"], d["dk"], d["dwq"], d["dwk"]
    pos = [s["coords"][:, 1 + a:2 + a].expand(-1, m) for a, m in enumerate(s["sections"])]
    angle = torch.cat(pos, 1).float() * s["freq"]
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    out, grads, dws = [], [], []
    for x, w, name in ((q, s["wq"], "dq"), (k, s["wk"], "dk")):
        x = x.float()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        y = x * r * w
        out.append(_turn(y, cos, sin).to(q.dtype))
        if c["train"]:
            a = _turn(s[name].float(), cos, -sin)
            dws.append((a * x * r).sum((0, 1)))
            a = a * w
            m = (a * x).mean(-1, keepdim=True)
            grads.append((r * a - r * r * r * m * x).to(q.dtype))
    return tuple(out + grads + dws)


def _turn(x, cos, sin):
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)


def _run_attend(s):
    c = s["case"]
    H, K, D = c["heads"], c["kv"], c["dim"]
    q, k, v = _parts(s["qkv"], H, K, D)
    if own:
        import paper_1505_02890_amd as scn
        how = dict(left=_bound(c["left"]), right=_bound(c["right"]), sinks=c["sinks"])
        o, lse = scn.attn_fwd(q, k, v, s["ranges"], **how)
        if not c["train"]:
            return o, lse
        d = scn.attn_bwd(q, k, v, o, lse, s["do"], s["ranges"], **how)
        return o, lse, d["dq"], d["dk"], d["dv"]
    q, k, v = (t.float().transpose(0, 1).contiguous() for t in (q, k, v))  # [heads][rows][D]
    G, n, scale = H // K, c["rows"], 1.0 / math.sqrt(D)
    o = torch.empty(H, n, D, device="cuda")
    lse = torch.empty(H, n, device="cuda")
    if c["train"]:
        do = s["do"].float().transpose(0, 1).contiguous()
        dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    at = 0
    for m in s["lens"]:
        step = max(64, min(1024, (1 << 24) // max(1, m * H)))
        for i0 in range(0, m, step):
            i1 = min(m, i0 + step)
            lo, hi, keys, see = _visible(i0, i1, m, c)
            nf = keys.numel() - (hi - lo)  # sinks before the window's first key

            def rows(t):
                w = t[:, at + lo:at + hi]
                return torch.cat([t[:, at:at + nf], w], 1) if nf else w
            kk, vv = rows(k), rows(v)
            Q = q[:, at + i0:at + i1].reshape(K, G * (i1 - i0), D)
            x = torch.bmm(Q, kk.transpose(1, 2)) * scale
            x = x.view(K, G, i1 - i0, -1).masked_fill_(~see, -math.inf)
            top = x.amax(-1, keepdim=True)
            p = (x - top).exp_()
            z = p.sum(-1, keepdim=True)
            p = (p / z).view(K, G * (i1 - i0), -1)
            O = torch.bmm(p, vv)
            o[:, at + i0:at + i1] = O.view(H, i1 - i0, D)
            lse[:, at + i0:at + i1] = (top + z.log()).view(H, i1 - i0)
            if c["train"]:
                dO = do[:, at + i0:at + i1].reshape(K, G * (i1 - i0), D)
                delta = (dO * O).sum(-1, keepdim=True)
                ds = p * (torch.bmm(dO, vv.transpose(1, 2)) - delta) * scale
                dq[:, at + i0:at + i1] = torch.bmm(ds, kk).view(H, i1 - i0, D)
                dkk, dvv = torch.bmm(ds.transpose(1, 2), Q), torch.bmm(p.transpose(1, 2), dO)
                for t, u in ((dk, dkk), (dv, dvv)):
                    t[:, at:at + nf] += u[:, :nf]
                    t[:, at + lo:at + hi] += u[:, nf:]
        at += m

    def done(t):
        return t.transpose(0, 1).to(s["qkv"].dtype).contiguous()
    if not c["train"]:
        return done(o), lse
    return done(o), lse, done(dq), done(dk), done(dv)


def _visible(i0, i1, m, c):
    """Keys that sites [i0, i1) of a sample of m see: the window's range [lo, hi), all keys
    (sinks that lie before the range first), and which site sees which."""
    left, right, sinks = c["left"], c["right"], c["sinks"]
    lo = 0 if left < 0 else max(0, i0 - left)
    hi = m if right < 0 else min(m, i1 + right)
    keys = torch.arange(lo, hi, device="cuda")
    if lo > 0 and sinks > 0:
        keys = torch.cat([torch.arange(0, min(sinks, lo), device="cuda"), keys])
    i = torch.arange(i0, i1, device="cuda")[:, None]
    see = torch.ones(i1 - i0, keys.numel(), dtype=torch.bool, device="cuda")
    if right >= 0:
        see &= keys <= i + right
    if left >= 0:
        see &= (keys >= i - left) | (keys < sinks)
    return lo, hi, keys, see


def _run_step(s):
    c = s["case"]
    B, C, H, K, D = (c[n] for n in ("streams", "capacity", "heads", "kv", "dim"))
    q, k, v = _parts(s["new"], H, K, D)
    if own:
        import paper_1505_02890_amd as scn
        o = scn.attn_step(q, k, v, s["k_cache"], s["v_cache"], s["length"],
                          left=_bound(c["left"]), sinks=c["sinks"])
        return o, s["k_cache"], s["v_cache"]
    ring = C - c["sinks"]
    reach = ring - 1 if c["left"] < 0 else min(c["left"], ring - 1)
    p = s["length"].long()[:, None]
    slot = torch.where(p < c["sinks"], p, c["sinks"] + (p - c["sinks"]) % ring)[:, 0]
    b = torch.arange(B, device="cuda")
    s["k_cache"][b, slot] = k
    s["v_cache"][b, slot] = v
    # the position that each slot holds: the last one that falls on it
    i = torch.arange(C, device="cuda")[None]
    held = torch.where(i < c["sinks"], i, p - (p - i) % ring)
    see = (held <= p) & ((i < c["sinks"]) | ((held >= c["sinks"]) & (held >= p - reach)))
    Q = q.float().reshape(B, K, H // K, D)
    kk = s["k_cache"].float().permute(0, 2, 3, 1).contiguous()
    x = torch.matmul(Q, kk) / math.sqrt(D)
    x = x.masked_fill_(~see[:, None, None], -math.inf)
    x = (x - x.amax(-1, keepdim=True)).exp_()
    x = x / x.sum(-1, keepdim=True)
    o = torch.matmul(x, s["v_cache"].float().permute(0, 2, 1, 3).contiguous())
    return o.reshape(B, H, D).to(q.dtype), s["k_cache"], s["v_cache"]


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def _pairs(case):
    """Visible (site, site) pairs, over the samples."""
    left, right, sinks = case["left"], case["right"], case["sinks"]
    tot = 0
    for m in _lengths(case):
        if m == 0:
            continue
        i = torch.arange(m)
        hi = torch.full_like(i, m) if right < 0 else torch.clamp(i + right + 1, max=m)
        lo = torch.zeros_like(i) if left < 0 else torch.clamp(i - left, min=0)
        tot += int((hi - lo).sum() + torch.minimum(lo, torch.full_like(i, sinks)).sum())
    return tot


def work(case):
    H, K, D = case["heads"], case["kv"], case["dim"]
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rotate":
        n = case["rows"]
        x = n * (H + K) * D
        byt = 2 * x * e + n * 4 * (case["ndim"] + 1) + 2 * D * 4
        fl = 8 * x
        if case["train"]:
            byt += 2 * x * e + 2 * D * 4  # the gradients in and out
            fl += 16 * x
        return dict(bytes=byt, flops=fl)
    if case["op"] == "attend":
        n, p = case["rows"], _pairs(case)
        byt = n * ((2 * H + 2 * K) * D * e + 4 * H)
        fl = 4 * D * H * p
        if case["train"]:
            byt += n * (2 * H + 2 * K) * D * e  # do in; dq, dk, dv out
            fl += 10 * D * H * p
        return dict(bytes=byt, flops=fl)
    B, C = case["streams"], case["capacity"]
    ring = C - case["sinks"]
    see = case["sinks"] + (ring if case["left"] < 0 else min(case["left"] + 1, ring))
    # streams of any age up to three times the capacity see about a sixth less
    part = 1.0 if case["full"] else 1.0 - see / (6.0 * C)
    return dict(bytes=int(B * ((2 * see * K * part + 2 * H + 4 * K) * D * e)),
                flops=int(4 * B * H * see * part * D))


# --------------------------------------------------------------------------
# the definition, in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "attend": _exact_attend, "step": _exact_step}[case["op"]](s)


def _exact_rotate(s):
    c = s["case"]
    n, H, K, D = c["rows"], c["heads"], c["kv"], c["dim"]
    axis = [a for a, m in enumerate(s["sections"]) for _ in range(m)]
    angle = s["coords"][:, [1 + a for a in axis]].double() * s["freq"].double()
    unit = torch.polar(torch.ones_like(angle), angle)[:, None, :]  # e^(i angle)
    x = s["qkv"].double().view(n, H + 2 * K, D)
    outs, dxs, dws = [], [], []
    for lo, hi, w, dy in ((0, H, s["wq"], s.get("dq")), (H, H + K, s["wk"], s.get("dk"))):
        xx, ww = x[:, lo:hi], w.double()
        norm = ((xx ** 2).sum(-1, keepdim=True) / D + EPS).sqrt()
        u = xx / norm
        z = torch.view_as_complex((u * ww).reshape(n, hi - lo, D // 2, 2).contiguous())
        outs.append(torch.view_as_real(z * unit).reshape(n, hi - lo, D))
        if c["train"]:
            gz = torch.view_as_complex(dy.double().reshape(n, hi - lo, D // 2, 2).contiguous())
            gy = torch.view_as_real(gz * unit.conj()).reshape(n, hi - lo, D)
            dws.append((gy * u).sum(1).sum(0))
            gu = gy * ww
            dxs.append((gu - u * (gu * u).sum(-1, keepdim=True) / D) / norm)
    return tuple(outs + dxs + dws)


def _exact_attend(s):
    c = s["case"]
    n, H, K, D = c["rows"], c["heads"], c["kv"], c["dim"]
    x = s["qkv"].view(n, H + 2 * K, D)
    o = torch.empty(n, H, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(H, n, dtype=torch.float64, device="cuda")
    if c["train"]:
        dx = torch.zeros(n, H + 2 * K, D, dtype=torch.float64, device="cuda")
    at = 0
    for m in s["lens"]:
        if m == 0:
            continue
        j = torch.arange(m, device="cuda")
        for i0 in range(0, m, 4096):
            i = torch.arange(i0, min(m, i0 + 4096), device="cuda")
            gap = j[None, :] - i[:, None]
            hide = torch.zeros_like(gap, dtype=torch.bool)
            if c["left"] >= 0:
                hide |= (gap < -c["left"]) & (j >= c["sinks"])[None, :]
            if c["right"] >= 0:
                hide |= gap > c["right"]
            r = slice(at + i0, at + i0 + len(i))
            for h in range(H):
                hk, hv = H + h * K // H, H + K + h * K // H
                kd, vd = x[at:at + m, hk].double(), x[at:at + m, hv].double()
                qd = x[r, h].double()
                w = qd @ kd.T
                w /= D ** 0.5
                w[hide] = -math.inf
                lse[h, r] = torch.logsumexp(w, 1)
                w -= lse[h, r][:, None]
                w.exp_()
                o[r, h] = w @ vd
                if c["train"]:
                    g = s["do"][r, h].double()
                    dx[at:at + m, hv] += w.T @ g
                    dw = g @ vd.T
                    dw -= (g * o[r, h]).sum(1, keepdim=True)
                    dw *= w
                    dw /= D ** 0.5
                    dx[r, h] += dw @ kd
                    dx[at:at + m, hk] += dw.T @ qd
        at += m
    if not c["train"]:
        return o, lse
    return o, lse, dx[:, :H], dx[:, H:H + K], dx[:, H + K:]


def _exact_step(s):
    c = s["case"]
    B, C, H, K, D = (c[n] for n in ("streams", "capacity", "heads", "kv", "dim"))
    x = s["new"].view(B, H + 2 * K, D)
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    o = torch.empty(B, H, D, dtype=torch.float64, device="cuda")
    S = c["sinks"]
    ring = C - S
    reach = ring - 1 if c["left"] < 0 else min(c["left"], ring - 1)
    for b, p in enumerate(s["length"].tolist()):
        now = p if p < S else S + (p - S) % ring
        kc[b, now] = x[b, H:H + K].double()
        vc[b, now] = x[b, H + K:].double()
        first = list(range(0, min(S, p + 1)))
        rest = torch.arange(min(max(S, p - reach), p + 1), p + 1, device="cuda")
        slots = torch.cat([torch.tensor(first, dtype=torch.long, device="cuda"),
                           S + (rest - S) % ring])
        kk, vv = kc[b, slots], vc[b, slots]
        for h in range(H):
            w = torch.softmax(kk[:, h * K // H] @ x[b, h].double() / D ** 0.5, 0)
            o[b, h] = w @ vv[:, h * K // H]
    return o, kc, vc
