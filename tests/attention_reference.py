"""Plain 64-bit references of the attention operators (numpy, one sample and head at
a time), each with a bound on how far a result may be off.

The bounds follow from the arithmetic.  u is half a unit of the result's type (2^-8
for bf16, 2^-24 for fp32) and e = 2^-24.
* Scores: a sum of D products, held in fp32, is within D e sum |q||k| of its value
  (n roundings of a sum of n terms); fp32 operands are split into three bf16 values
  with a rest of at most 2^-24 of each product more.  Each weight p = exp(s - lse) is
  then off by the errors of its score and of lse, and of exp2 and its argument:
  at most es = 2 (D + 2) e scale sum|q||k| + (|s| + |lse| + 8) 4 e, relatively.
* bf16: p, and ds in the gradients, are rounded to bf16 before their products, which
  costs u of each term; o is read back rounded by the backward, which moves
  <do, o> by u sum |do||o|.
* Sums of m terms in fp32 add at most m e of the terms' absolute sum; the kernels' sums
  are trees of a few dozen products a step, so sqrt(m) + 64 stands for m.
"""
from __future__ import annotations

import numpy as np

E = 2.0 ** -24


def unit(bf16: bool) -> float:
    return 2.0 ** -8 if bf16 else E


def visible(m, left, right, sinks):
    i, j = np.arange(m)[:, None], np.arange(m)[None]
    see = np.ones((m, m), bool)
    if right is not None:
        see &= j <= i + right
    if left is not None:
        see &= (j >= i - left) | (j < sinks)
    return see


def attention(q, k, v, lens, left, right, sinks, scale, bf16, do=None):
    """q [n, Hq, D], k, v [n, Hk, D] in float64.  Returns {name: (value, bound)}."""
    n, H, D = q.shape
    K = k.shape[1]
    u = unit(bf16)
    out = {"o": np.zeros((n, H, D)), "lse": np.zeros((H, n))}
    if do is not None:
        out.update(dq=np.zeros((n, H, D)), dk=np.zeros((n, K, D)), dv=np.zeros((n, K, D)))
    tol = {x: np.zeros_like(a) for x, a in out.items()}
    at = 0
    for m in lens:
        r = slice(at, at + m)
        at += m
        if m == 0:
            continue
        see = visible(m, left, right, sinks)
        sums = (np.sqrt(m) + 64) * E
        for h in range(H):
            g = h // (H // K)
            Q, KK, V = q[r, h], k[r, g], v[r, g]
            s = np.where(see, scale * (Q @ KK.T), -np.inf)
            top = s.max(1, keepdims=True)
            w = np.exp(s - top)
            z = w.sum(1, keepdims=True)
            p = w / z
            lse = top + np.log(z)
            mag = scale * (np.abs(Q) @ np.abs(KK).T)
            es = np.where(see, 2 * (D + 2) * E * mag + (np.abs(s) + np.abs(lse) + 8) * 4 * E, 0)
            es = np.where(see, es, 0).max(1, keepdims=True)  # lse's own share too
            A = p @ np.abs(V)
            out["o"][r, h] = p @ V
            tol["o"][r, h] = ((u if bf16 else 0) + 2 * es + 2 * sums) * A + 1.01 * u * np.abs(
                out["o"][r, h])
            out["lse"][h, r] = lse[:, 0]
            tol["lse"][h, r] = (2 * es + sums + 2 * E * np.abs(lse) + 4 * E)[:, 0]
            if do is None:
                continue
            G = do[r, h]
            o = out["o"][r, h]
            delta = (G * o).sum(1, keepdims=True)
            dp = G @ V.T
            ds = p * (dp - delta)
            # error of ds: p's, dp's and delta's (which takes o as the forward rounded it)
            ed = (np.abs(G) * tol["o"][r, h]).sum(1, keepdims=True) + (
                D + 2) * E * (np.abs(G) * np.abs(o)).sum(1, keepdims=True)
            edp = 2 * (D + 2) * E * (np.abs(G) @ np.abs(V).T)
            eds = 3 * es * np.abs(ds) + p * (ed + edp + 2 * E * (np.abs(dp) + np.abs(delta)))
            eds = eds + (1.01 * u if bf16 else 0) * (np.abs(ds) + eds)
            ep = p * (3 * es + (1.01 * u if bf16 else 0))
            out["dq"][r, h] = scale * (ds @ KK)
            tol["dq"][r, h] = scale * ((eds + 2 * sums * np.abs(ds)) @ np.abs(KK))
            out["dk"][r, g] += scale * (ds.T @ Q)
            tol["dk"][r, g] += scale * ((eds + 2 * sums * np.abs(ds)).T @ np.abs(Q))
            out["dv"][r, g] += p.T @ G
            tol["dv"][r, g] += (ep + 2 * sums * p).T @ np.abs(G)
    for x in ("dq", "dk", "dv"):
        if x in out:
            tol[x] += 1.01 * u * (np.abs(out[x]) + tol[x])
    return {x: (out[x], tol[x] + 1e-30) for x in out}


def step(q, k, v, kc, vc, length, left, sinks, scale, bf16):
    """One step of every stream: (o, bound), the caches updated in place."""
    B, H, D = q.shape
    K, cap = k.shape[1], kc.shape[1]
    ring = cap - sinks
    reach = ring - 1 if left is None else min(left, ring - 1)
    u = unit(bf16)
    o, tol = np.zeros((B, H, D)), np.zeros((B, H, D))
    for b in range(B):
        p = max(0, int(length[b]))
        slot = [j if j < sinks else sinks + (j - sinks) % ring for j in range(p + 1)
                if j < sinks or j >= p - reach]
        kc[b, slot[-1]], vc[b, slot[-1]] = k[b], v[b]
        for h in range(H):
            g = h // (H // K)
            KK, V = kc[b, slot, g], vc[b, slot, g]
            s = scale * (KK @ q[b, h])
            w = np.exp(s - s.max())
            w /= w.sum()
            es = 2 * (D + 2) * E * scale * (np.abs(KK) @ np.abs(q[b, h])).max() + (
                2 * np.abs(s).max() + 8) * 4 * E
            o[b, h] = w @ V
            tol[b, h] = (2 * es + 2 * (np.sqrt(len(slot)) + 64) * E) * (w @ np.abs(
                V)) + 1.01 * u * np.abs(o[b, h])
    return o, tol + 1e-30


def norm_rotate(x, w, coords, freq, sections, eps, bf16, dy=None):
    """x [n, H, D] in float64.  Returns (y, bound) or (y, bound, dx, bound, dw, bound).
    Norm and angles are within (D + 16) e relatively; a turn mixes the pair."""
    n, H, D = x.shape
    u = unit(bf16)
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    ang = np.zeros((n, D // 2))
    for j, a in enumerate(axis):
        ang[:, j] = coords[:, 1 + a].astype(np.float64) * float(freq[j])
    cs, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
    w = np.ones(D) if w is None else w

    def turn(z, c, s):
        a, b = z[..., 0::2], z[..., 1::2]
        return np.stack([a * c - b * s, a * s + b * c], -1).reshape(z.shape)

    def pair(z):  # |a| + |b| for each of a pair
        t = np.abs(z[..., 0::2]) + np.abs(z[..., 1::2])
        return np.repeat(t, 2, -1)

    rel = (D + 16) * E
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    t = x * r * w
    y = turn(t, cs, sn)
    ty = rel * pair(t) + 1.01 * u * np.abs(y) + 1e-30
    if dy is None:
        return y, ty
    g = turn(dy, cs, -sn)
    eg = 8 * E * pair(dy)
    a = g * w
    mean = (a * x).mean(-1, keepdims=True)
    em = ((eg * np.abs(w * x)) + D * E * np.abs(a * x)).mean(-1, keepdims=True)
    dx = r * a - r ** 3 * x * mean
    tx = r * (eg * np.abs(w) + rel * np.abs(a)) + r ** 3 * np.abs(x) * (
        em + 3 * rel * np.abs(mean)) + 1.01 * u * np.abs(dx) + 1e-30
    dw = (g * x * r).sum((0, 1))
    tw = ((eg + (rel + (np.sqrt(n * H) + 64) * E) * np.abs(g)) * np.abs(x) * r).sum((0, 1)) + 1e-30
    return y, ty, dx, tx, dw, tw
