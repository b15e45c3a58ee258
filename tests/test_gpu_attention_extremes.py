"""Attention of values far from 1: scores past 2^31, values near the type's largest,
fp32 operands whose split has no low parts, and infinities that a row sees."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import attention_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E = ref.E


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


def f64(t):
    torch.cuda.synchronize()
    return t.detach().double().cpu().numpy()


def bounds(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def check(name, got, want, tol):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    with np.errstate(invalid="ignore"):  # inf - inf
        near = np.abs(got - want) <= tol
    bad = ~(near | (got == want) | (np.isnan(got) & np.isnan(want)))
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{name}: {bad.sum()}/{bad.size} outside their bound, the first at "
                             f"{i}: {got[i]!r} against {want[i]!r}, bound {tol[i]:.3g}")


# --------------------------------------------------------------------------
# large scores
# --------------------------------------------------------------------------
# Entries are whole numbers times powers of two, so every score is exact in fp32 and a row's
# largest ones are equal or 2^e / 4 and more apart: the weights are 1 / (how many are
# largest) and 0, whatever e is.  Bounds are those of attention_reference with the weights'
# own error es left at 16 roundings (of the exponential, the sum, its logarithm and
# their differences), and of <do, o> 2^-15 as where a row sees one key.  The gradients form
# the weights from log sums in fp32: each is within 3 roundings of it (its own, its
# product's and the difference's) of its value, which past 8192 would be more than 2^-9.
# From there on the gradients must not depend on it.

def whole(n, heads, D, seed, exponent, dtype):
    rng = np.random.default_rng(seed)
    x = rng.integers(-3, 4, (n, heads, D)) * 2.0 ** exponent
    return torch.tensor(x, dtype=torch.float32).to(TYPES[dtype]).cuda()


def one_hot(q, k, v, lens, see, scale, bf16, do):
    n, H, D = q.shape
    K = k.shape[1]
    u = ref.unit(bf16)
    val = {"o": np.zeros((n, H, D)), "lse": np.zeros((H, n)), "dq": np.zeros((n, H, D)),
           "dk": np.zeros((n, K, D)), "dv": np.zeros((n, K, D))}
    tol = {x: np.zeros_like(a) for x, a in val.items()}
    at = 0
    for m in lens:
        r = slice(at, at + m)
        at += m
        es, sums = 16 * E, (np.sqrt(m) + 64) * E
        for h in range(H):
            g = h // (H // K)
            Q, KK, V, G = q[r, h], k[r, g], v[r, g], do[r, h]
            s = np.where(see(m), scale * (Q @ KK.T), -np.inf)
            top = s.max(1, keepdims=True)
            w = np.exp(s - top)
            z = w.sum(1, keepdims=True)
            p = w / z
            o = p @ V
            val["o"][r, h] = o
            tol["o"][r, h] = ((u if bf16 else 0) + es + sums) * (p @ np.abs(V)) + u * np.abs(o)
            val["lse"][h, r] = (top + np.log(z))[:, 0]
            tol["lse"][h, r] = (4 * E * np.abs(top) + es)[:, 0]
            dp = G @ V.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            mag = np.abs(G) @ np.abs(V).T
            eg = es + np.where(np.abs(top) > 8192, 0, 3 * E * (np.abs(top) + np.log(z)))
            eds = eg * np.abs(ds) + p * 2.0 ** -15 * (mag + (p * mag).sum(1, keepdims=True))
            eds = eds + (u if bf16 else 0) * (np.abs(ds) + eds)
            ep = p * (eg + sums + (u if bf16 else 0))
            val["dq"][r, h] = scale * (ds @ KK)
            tol["dq"][r, h] = scale * (eds + sums * np.abs(ds)) @ np.abs(KK)
            val["dk"][r, g] += scale * (ds.T @ Q)
            tol["dk"][r, g] += scale * (eds + sums * np.abs(ds)).T @ np.abs(Q)
            val["dv"][r, g] += p.T @ G
            tol["dv"][r, g] += ep.T @ np.abs(G)
    for x in ("dq", "dk", "dv"):
        tol[x] += u * (np.abs(val[x]) + tol[x])
    return val, {x: t + 1e-30 for x, t in tol.items()}  # (fp32 ends at 1e-45)


EXPONENTS = [0, 8, 13, 20, 31, 40, 90]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("exponent", EXPONENTS)
@pytest.mark.parametrize("D,lens,left,right,sinks", [
    (32, [130, 1, 70], None, None, 0), (64, [300, 41], 60, 3, 2), (128, [200], None, 0, 0)])
def test_scores_past_the_exponent(scn, dtype, exponent, D, lens, left, right, sinks):
    n, H, K, scale = sum(lens), 4, 2, 0.25
    q = whole(n, H, D, 1, exponent - exponent // 2, dtype)
    k = whole(n, K, D, 2, exponent // 2, dtype)
    g = torch.Generator().manual_seed(3)
    v, do = (torch.randn(n, h, D, generator=g).to(TYPES[dtype]).cuda() for h in (K, H))
    how = dict(left=left, right=right, sinks=sinks, scale=scale)
    o, lse = scn.attn_fwd(q, k, v, bounds(lens), **how)
    want, tol = one_hot(f64(q), f64(k), f64(v), lens,
                        lambda m: ref.visible(m, left, right, sinks), scale, dtype == "bf16",
                        f64(do))
    check("o", o, want["o"], tol["o"])
    check("lse", lse, want["lse"], tol["lse"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("exponent", EXPONENTS)
@pytest.mark.parametrize("D,lens,left,right,sinks", [
    (32, [130, 1, 70], None, None, 0), (64, [300, 41], 60, 3, 2), (128, [200], None, 0, 0),
    (32, [400], 10, 0, 2)])
def test_gradients_of_scores_past_the_exponent(scn, dtype, exponent, D, lens, left, right, sinks):
    n, H, K, scale = sum(lens), 4, 2, 0.25
    q = whole(n, H, D, 1, exponent - exponent // 2, dtype)
    k = whole(n, K, D, 2, exponent // 2, dtype)
    g = torch.Generator().manual_seed(3)
    v, do = (torch.randn(n, h, D, generator=g).to(TYPES[dtype]).cuda() for h in (K, H))
    how = dict(left=left, right=right, sinks=sinks, scale=scale)
    want, tol = one_hot(f64(q), f64(k), f64(v), lens,
                        lambda m: ref.visible(m, left, right, sinks), scale, dtype == "bf16",
                        f64(do))
    # o and lse as a forward rounds them
    o = torch.tensor(want["o"], dtype=torch.float32).to(TYPES[dtype]).cuda()
    lse = torch.tensor(want["lse"], dtype=torch.float32).cuda()
    d = scn.attn_bwd(q, k, v, o, lse, do, bounds(lens), **how)
    for x in ("dq", "dk", "dv"):
        check(x, d[x], want[x], tol[x])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("exponent", EXPONENTS)
@pytest.mark.parametrize("H,K,D,cap,length", [(4, 2, 64, 300, 299), (3, 1, 40, 5000, 4998),
                                              (1, 1, 128, 40, 0)])
def test_steps_of_scores_past_the_exponent(scn, dtype, exponent, H, K, D, cap, length):
    q = whole(1, H, D, 1, exponent - exponent // 2, dtype)
    kc = whole(cap, K, D, 2, exponent // 2, dtype)
    k = whole(1, K, D, 4, exponent // 2, dtype)
    g = torch.Generator().manual_seed(3)
    vc, v = (torch.randn(m, K, D, generator=g).to(TYPES[dtype]).cuda() for m in (cap, 1))
    o = scn.attn_step(q, k, v, kc[None], vc[None],
                      torch.tensor([length], dtype=torch.int32, device="cuda"), scale=0.25)
    m = length + 1
    s = 0.25 * np.einsum("hd,mhd->hm", f64(q)[0], np.repeat(f64(kc)[:m], H // K, 1))
    w = np.exp(s - s.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    V = np.repeat(f64(vc)[:m], H // K, 1)
    u = ref.unit(dtype == "bf16")
    want, mag = np.einsum("hm,mhd->hd", w, V), np.einsum("hm,mhd->hd", w, np.abs(V))
    check("o", o, want[None], ((16 + np.sqrt(m) + 64) * E * mag + u * np.abs(want))[None])


# --------------------------------------------------------------------------
# values near the type's largest: weights are at most 1, but their terms before the
# division by their sum need not be
# --------------------------------------------------------------------------

def large_values(n, heads, D, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    x = (0.8 + 0.1 * torch.rand(n, heads, D, generator=g)) * torch.finfo(TYPES[dtype]).max
    x[:, :, 1::2] *= -1
    return x.to(TYPES[dtype]).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_values_near_the_largest(scn, dtype, D):
    lens, H, K = [200, 1, 33], 2, 1
    n = sum(lens)
    g = torch.Generator().manual_seed(5)
    q, k = (torch.randn(n, h, D, generator=g).to(TYPES[dtype]).cuda() for h in (H, K))
    v = large_values(n, K, D, 6, dtype)
    o, lse = scn.attn_fwd(q, k, v, bounds(lens), right=0)
    want = ref.attention(f64(q), f64(k), f64(v), lens, None, 0, 0, D ** -0.5, dtype == "bf16")
    check("o", o, *want["o"])
    check("lse", lse, *want["lse"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,cap,length", [(64, 200, 199), (40, 5000, 4999)])
def test_steps_of_values_near_the_largest(scn, dtype, D, cap, length):
    H, K = 4, 2
    g = torch.Generator().manual_seed(7)
    q, k, kc = (torch.randn(m, h, D, generator=g).to(TYPES[dtype]).cuda()
                for m, h in ((1, H), (1, K), (cap, K)))
    v, vc = large_values(1, K, D, 8, dtype), large_values(cap, K, D, 9, dtype)
    want, tol = ref.step(f64(q), f64(k), f64(v), f64(kc)[None], f64(vc)[None], [length], None, 0,
                         D ** -0.5, dtype == "bf16")
    o = scn.attn_step(q, k, v, kc[None], vc[None],
                      torch.tensor([length], dtype=torch.int32, device="cuda"))
    check("o", o, want, tol)


# --------------------------------------------------------------------------
# infinities and NaN that a row sees
# --------------------------------------------------------------------------

def one_row(q, K, V, scale, bf16):
    """o [H, D] of one query row on K, V [m, H, D], and its bound: channels that an infinite
    value enters are infinite, rows with a score of +inf or NaN are NaN, and scores of -inf
    have no weight."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = scale * np.einsum("hd,mhd->hm", q, K)
        top = s.max(1, keepdims=True)
        w = np.exp(s - top)
        w /= w.sum(1, keepdims=True)
        live = (w != 0)[..., None]
        Vt = V.transpose(1, 0, 2)
        terms = np.where(live, w[..., None] * Vt, 0)
        o = terms.sum(1)
        fin = np.where(np.isfinite(terms), terms, 0)
        smag = scale * np.einsum("hd,mhd->hm", np.abs(q), np.where(np.isfinite(K), np.abs(K), 0))
        es = 2 * (q.shape[1] + 2) * E * smag.max(1) + (
            2 * np.where(np.isfinite(s), np.abs(s), 0).max(1) + 8) * 4 * E
    u = ref.unit(bf16)
    m = K.shape[0]
    tol = ((2 * es)[:, None] + 2 * (np.sqrt(m) + 64) * E + (u if bf16 else 0)) * np.abs(
        fin).sum(1) + 1.01 * u * np.abs(np.where(np.isfinite(o), o, 0)) + 1e-30
    return o, tol


INF = float("inf")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [24, 40, 64, 80, 128])
@pytest.mark.parametrize("cap,at", [(50, 49), (50, 10), (4000, 1234), (4000, 3999)])
@pytest.mark.parametrize("what", ["inf", "-inf", "both", "nan", "key"])
def test_steps_see_infinities(scn, dtype, D, cap, at, what):
    H = K = 2
    t = TYPES[dtype]
    g = torch.Generator().manual_seed(11)
    q, kc, vc = (torch.randn(m, h, D, generator=g).to(t).cuda()
                 for m, h in ((1, H), (cap, K), (cap, K)))
    if what == "key":  # an infinite first channel: no weight for the first head, NaN for the other
        kc[at, :, 0] = -torch.sign(q[0, :, 0]) * INF
        kc[at, 1, 0] *= -1
    elif what == "both":  # of both signs in one channel
        vc[at, :, 3], vc[at // 2, :, 3] = INF, -INF
    else:
        vc[at, :, 3] = {"inf": INF, "-inf": -INF, "nan": float("nan")}[what]
        vc[at, 0, D - 1] = -INF
    want, tol = one_row(f64(q)[0], f64(kc), f64(vc), D ** -0.5, dtype == "bf16")
    k, v = kc[cap - 1:].clone(), vc[cap - 1:].clone()  # the new token's
    o = scn.attn_step(q, k, v, kc[None], vc[None],
                      torch.tensor([cap - 1], dtype=torch.int32, device="cuda"))
    check("o", o, want[None], tol[None])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [24, 64, 80, 128])
@pytest.mark.parametrize("what", ["inf", "both", "key"])
def test_rows_see_infinities(scn, dtype, D, what):
    n, at = 150, 70
    t = TYPES[dtype]
    g = torch.Generator().manual_seed(12)
    q, k, v = (torch.randn(n, 2, D, generator=g).to(t).cuda() for _ in range(3))
    if what == "key":
        k[at, :, 0] = -INF
    else:
        v[at, :, 3] = INF
        if what == "both":
            v[at // 2, 0, 3] = -INF
    o, _ = scn.attn_fwd(q, k, v, bounds([n]), right=0)
    Q, KK, V, got = f64(q), f64(k), f64(v), f64(o)
    for i in (0, at // 2, at - 1, at, at + 1, n - 1):
        want, tol = one_row(Q[i], KK[:i + 1], V[:i + 1], D ** -0.5, dtype == "bf16")
        check(f"o[{i}]", got[i], want, tol)


# --------------------------------------------------------------------------
# fp32 values whose parts in bf16 end early: bf16 holds nothing below 2^-133, so a value of
# 2^-112 keeps 21 bits of 24, and one of 2^-125 eight
# --------------------------------------------------------------------------

@pytest.mark.parametrize("power", [-112, -120, -124])
@pytest.mark.parametrize("D,lens,left,right,sinks", [
    (32, [130, 1, 70], None, 0, 0), (64, [300, 41], 60, 3, 2), (128, [200], None, None, 0),
    (24, [400], 10, 0, 2)])
def test_tiny_values_keep_their_bits(scn, D, lens, left, right, sinks, power):
    # values and gradients scaled by a power of two: results scale with them (but for what
    # lies below the smallest fp32)
    n, H, K = sum(lens), 2, 1
    up, floor = 2.0 ** -power, 2.0 ** -149 * 2.0 ** -power
    g = torch.Generator().manual_seed(14)
    q, k = (torch.randn(n, h, D, generator=g).cuda() for h in (H, K))
    v = torch.randn(n, K, D, generator=g)
    do = torch.randn(n, H, D, generator=g).cuda()
    small = (v.double() * 2.0 ** power).float()
    how = dict(left=left, right=right, sinks=sinks)
    o, _ = scn.attn_fwd(q, k, small.cuda(), bounds(lens), **how)
    args = (lens, left, right, sinks, D ** -0.5, False)
    want = ref.attention(f64(q), f64(k), small.double().numpy() * up, *args)
    check("o", f64(o) * up, want["o"][0], want["o"][1] + 2 * floor)
    o, lse = scn.attn_fwd(q, k, v.cuda(), bounds(lens), **how)
    less = (do.double() * 2.0 ** power).float()
    d = scn.attn_bwd(q, k, v.cuda(), o, lse, less, bounds(lens), **how)
    want = ref.attention(f64(q), f64(k), v.double().numpy(), *args, f64(less) * up)
    # every sum's terms are rounded to multiples of 2^-149: D of them in a dP, weighted by p,
    # one in its dS, and one a term in the result
    a, b = (np.abs(f64(t)).max() for t in (q, k))
    m = max(lens)
    extra = {"dv": H * m * floor, "dq": 2 * (b + 1) * (D + 2 + m) * floor,
             "dk": H * m * (a + 1) * (D + 3) * floor}
    for x in ("dq", "dk", "dv"):
        check(x, f64(d[x]) * up, want[x][0], want[x][1] + extra[x])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [24, 32, 64, 128])
@pytest.mark.parametrize("what", ["q", "k"])
def test_rows_of_nan_are_those_that_see_it(scn, dtype, D, what):
    # a query or a key of NaN: its rows, and the keys that they see, have no finite result; all
    # others have what they have without it
    m, H, K, left, sinks, at = 300, 2, 1, 40, 1, 100
    t = TYPES[dtype]
    g = torch.Generator().manual_seed(13)
    q, k, v, do = (torch.randn(m, h, D, generator=g).to(t).cuda() for h in (H, K, K, H))
    want = ref.attention(f64(q), f64(k), f64(v), [m], left, 0, sinks, D ** -0.5, dtype == "bf16",
                         f64(do))
    (q if what == "q" else k)[at] = float("nan")
    how = dict(left=left, right=0, sinks=sinks)
    o, lse = scn.attn_fwd(q, k, v, bounds([m]), **how)
    d = scn.attn_bwd(q, k, v, o, lse, do, bounds([m]), **how)
    i = np.arange(m)
    rows = (i == at) if what == "q" else (i >= at) & (i <= at + left)
    see = ref.visible(m, left, 0, sinks)
    keys = see[rows].any(0)
    for name, got, none in (("o", o, rows), ("dq", d["dq"], rows), ("dk", d["dk"], keys),
                            ("dv", d["dv"], keys)):
        got = f64(got)
        assert np.isnan(got[none]).all(), name
        check(name, got[~none], want[name][0][~none], want[name][1][~none])
    assert np.isnan(f64(lse)[:, rows]).all()
    check("lse", f64(lse)[:, ~rows], want["lse"][0][:, ~rows], want["lse"][1][:, ~rows])
