"""Plain 64-bit references of cross attention, the norms around a block and clipping
(numpy), each with a bound on how far a result may be off.

u is half a unit of the result's type (2^-8 for bf16, 2^-24 for fp32) and e = 2^-24.
Cross attention takes the bounds of ``attention_reference`` (its derivation holds for
any number of keys).  The norms:
* A sum of C terms in fp32 is within C e of the sum of their sizes, a mean's root
  half of that relatively, and the reciprocal root and the products around it add
  some units: n(t) is within N = (C / 2 + 8) e, relatively, where its input is exact.
* sigmoid is within 8 e (an exponential, a sum, a division and a product).
* y = alpha x + g u adds its own rounding and that of alpha x; n(y) sees y's error
  once for itself and once in the mean.
* Gradients add a second sum of C terms each; what cancels is bounded by the sizes of
  its terms.
"""
from __future__ import annotations

import numpy as np

import attention_reference as att

E = att.E


def cross(q, k, v, qlens, klens, scale, bf16, do=None):
    """q [n, Hq, D], k, v [m, Hk, D] in float64.  Returns {name: (value, bound)}."""
    n, H, D = q.shape
    m, K = k.shape[:2]
    shapes = {"o": (n, H, D), "lse": (H, n)}
    if do is not None:
        shapes.update(dq=(n, H, D), dk=(m, K, D), dv=(m, K, D))
    out = {x: np.zeros(s) for x, s in shapes.items()}
    tol = {x: np.full(s, 1e-30) for x, s in shapes.items()}
    out["lse"][:] = -np.inf
    q0 = k0 = 0
    for a, b in zip(qlens, klens):
        qs, ks = slice(q0, q0 + a), slice(k0, k0 + b)
        q0, k0 = q0 + a, k0 + b
        if a == 0 or b == 0:
            continue
        r = _rect(q[qs], k[ks], v[ks], scale, bf16, None if do is None else do[qs])
        for x, (value, bound) in r.items():
            at = {"o": qs, "dq": qs, "dk": ks, "dv": ks, "lse": (slice(None), qs)}[x]
            out[x][at], tol[x][at] = value, bound
    return {x: (out[x], tol[x]) for x in out}


def _rect(q, k, v, scale, bf16, do):
    """attention_reference.attention's formulas and bounds for one sample."""
    n, H, D = q.shape
    m, K = k.shape[:2]
    u = att.unit(bf16)
    out = {"o": np.zeros((n, H, D)), "lse": np.zeros((H, n))}
    if do is not None:
        out.update(dq=np.zeros((n, H, D)), dk=np.zeros((m, K, D)), dv=np.zeros((m, K, D)))
    tol = {x: np.zeros_like(a) for x, a in out.items()}
    sums, rows = (np.sqrt(m) + 64) * E, (np.sqrt(n * (H // K)) + 64) * E
    for h in range(H):
        g = h // (H // K)
        Q, KK, V = q[:, h], k[:, g], v[:, g]
        s = scale * (Q @ KK.T)
        top = s.max(1, keepdims=True)
        w = np.exp(s - top)
        z = w.sum(1, keepdims=True)
        p = w / z
        lse = top + np.log(z)
        es = (2 * (D + 2) * E * scale * (np.abs(Q) @ np.abs(KK).T)
              + (np.abs(s) + np.abs(lse) + 8) * 4 * E).max(1, keepdims=True)
        A = p @ np.abs(V)
        o = p @ V
        out["o"][:, h] = o
        eo = ((u if bf16 else 0) + 2 * es + 2 * sums) * A + 1.01 * u * np.abs(o)
        tol["o"][:, h] = eo + 1e-30
        out["lse"][h] = lse[:, 0]
        tol["lse"][h] = (2 * es + sums + 2 * E * np.abs(lse) + 4 * E)[:, 0]
        if do is None:
            continue
        G = do[:, h]
        delta = (G * o).sum(1, keepdims=True)
        dp = G @ V.T
        ds = p * (dp - delta)
        ed = (np.abs(G) * eo).sum(1, keepdims=True) + (D + 2) * E * (
            np.abs(G) * np.abs(o)).sum(1, keepdims=True)
        edp = 2 * (D + 2) * E * (np.abs(G) @ np.abs(V).T)
        eds = 3 * es * np.abs(ds) + p * (ed + edp + 2 * E * (np.abs(dp) + np.abs(delta)))
        eds = eds + (1.01 * u if bf16 else 0) * (np.abs(ds) + eds)
        ep = p * (3 * es + (1.01 * u if bf16 else 0))
        out["dq"][:, h] = scale * (ds @ KK)
        tol["dq"][:, h] = scale * ((eds + 2 * sums * np.abs(ds)) @ np.abs(KK))
        out["dk"][:, g] += scale * (ds.T @ Q)
        tol["dk"][:, g] += scale * ((eds + 2 * rows * np.abs(ds)).T @ np.abs(Q))
        out["dv"][:, g] += p.T @ G
        tol["dv"][:, g] += (ep + 2 * rows * p).T @ np.abs(G)
    for x in ("dq", "dk", "dv"):
        if x in out:
            tol[x] += 1.01 * u * (np.abs(out[x]) + tol[x]) + 1e-30
    return {x: (out[x], tol[x]) for x in out}


def sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z < 0, e, 1) / (1 + e)


def block(x, f, z, wf, wh, alpha, eps, res_bf16, bf16, dy=None, dh=None, h=True):
    """All [n, C] in float64 (f, z, wf, wh, dy, dh may be None).  Returns {name: (value,
    bound)} of y, h and, where dy or dh is given, of dx, df, dz, dwf, dwh."""
    n, C = x.shape
    ur, u = att.unit(res_bf16), att.unit(bf16)
    N = (C / 2 + 8) * E
    wf = np.ones(C) if wf is None else wf
    wh = np.ones(C) if wh is None else wh
    mean = lambda t: t.mean(1, keepdims=True)  # noqa: E731
    y, ey = alpha * x, 2 * E * np.abs(alpha * x)
    g = ge = 1.0
    if f is not None:
        rf = 1 / np.sqrt(mean(f * f) + eps)
        fn = f * rf
        if z is not None:
            g, ge = sigmoid(z), sigmoid(-z)
        part = g * wf * fn
        y = y + part
        ey = ey + (N + 12 * E) * np.abs(part) + E * np.abs(y)
    ry = 1 / np.sqrt(mean(y * y) + eps)
    yn = y * ry
    # n(y): its own rounding, y's error, and the mean's of it
    eyn = N * np.abs(yn) + ry * ey + np.abs(yn) * ry * mean(np.abs(yn) * ey)
    out = {"y": (y, ey + 1.01 * ur * np.abs(y)), "h": (yn * wh, eyn * np.abs(wh) + 1.01 * u * np.abs(
        yn * wh) + 2 * E * np.abs(yn * wh))}
    if dy is None and dh is None:
        return {a: (b, c + 1e-37) for a, (b, c) in out.items()}
    dY = np.zeros_like(x) if dy is None else dy
    eY = np.zeros_like(x)
    rows = (np.sqrt(n) + 64) * E  # sums over rows: trees of a few dozen terms a step
    if dh is not None:
        a = dh * wh
        m = mean(a * yn)
        em = mean(np.abs(a) * eyn) + (C + 4) * E * mean(np.abs(a * yn))
        er = N + ry * mean(np.abs(yn) * ey)  # of ry, relatively
        dY = dY + ry * (a - yn * m)
        eY = ry * (2 * E * np.abs(a) + eyn * np.abs(m) + np.abs(yn) * em) + (er + 4 * E) * ry * (
            np.abs(a) + np.abs(yn * m)) + E * np.abs(dY)
        out["dwh"] = ((dh * yn).sum(0), (np.abs(dh) * (eyn + (rows + 2 * E) * np.abs(yn))).sum(0))
    out["dx"] = (alpha * dY, abs(alpha) * eY + (1.01 * ur + 2 * E) * np.abs(alpha * dY))
    if f is not None:
        du = dY * g
        edu = eY * g + 10 * E * np.abs(du)
        b = du * wf
        eb = (edu + E * np.abs(du)) * np.abs(wf)
        m = mean(b * fn)
        em = mean(eb * np.abs(fn) + (N + (C + 4) * E) * np.abs(b * fn))
        out["df"] = (rf * (b - fn * m), rf * (eb + (N + 4 * E) * np.abs(b) + np.abs(fn) * (
            em + (2 * N + 4 * E) * np.abs(m))) + 1.01 * u * rf * np.abs(b - fn * m))
        out["dwf"] = ((du * fn).sum(0), ((edu + (N + rows) * np.abs(du)) * np.abs(fn)).sum(0))
        if z is not None:
            dz = dY * wf * fn * g * ge
            out["dz"] = (dz, eY * np.abs(wf * fn * g * ge) + (N + 24 * E + 1.01 * u) * np.abs(dz))
    return {a: (b, c + 1e-37) for a, (b, c) in out.items()}
