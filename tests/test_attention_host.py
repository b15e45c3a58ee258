"""CPU checks of attention among the active sites: the 64-bit references themselves
(brute force, differences, planted mistakes), and what the C ABI refuses before any
device work."""
from __future__ import annotations

import ctypes
import math
import os

import numpy as np
import pytest

import attention_reference as ref

P = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    from paper_1505_02890_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_1505_02890_amd.build import build
        build()
    return _lib.lib()


def data(n, H, K, D, seed):
    rng = np.random.default_rng(seed)
    return rng.standard_normal((n, H, D)), *(rng.standard_normal((n, K, D)) for _ in range(2))


def brute(q, k, v, lens, left, right, sinks, scale):
    """Attention term by term, from the header's words."""
    o = np.zeros_like(q)
    at = 0
    for m in lens:
        for i in range(m):
            for h in range(q.shape[1]):
                g = h // (q.shape[1] // k.shape[1])
                seen = [j for j in range(m) if (right is None or j <= i + right) and
                        (left is None or j >= i - left or j < sinks)]
                s = [scale * sum(q[at + i, h] * k[at + j, g]) for j in seen]
                z = sum(math.exp(x) for x in s)
                o[at + i, h] = sum(math.exp(x) / z * v[at + j, g] for x, j in zip(s, seen))
        at += m
    return o


@pytest.mark.parametrize("left,right,sinks", [(None, None, 0), (None, 0, 0), (3, 0, 0), (2, 1, 2),
                                              (0, 0, 1), (4, None, 5)])
def test_reference_equals_the_definition(left, right, sinks):
    lens = [7, 0, 1, 9]
    q, k, v = data(sum(lens), 4, 2, 8, 1)
    got = ref.attention(q, k, v, lens, left, right, sinks, 0.4, False)["o"][0]
    assert np.abs(got - brute(q, k, v, lens, left, right, sinks, 0.4)).max() < 1e-13


def test_reference_gradients_against_differences():
    lens, how = [8, 5], (3, 1, 1, 0.5, False)
    q, k, v = data(13, 2, 1, 8, 2)
    do = np.random.default_rng(3).standard_normal(q.shape)
    out = ref.attention(q, k, v, lens, *how, do)
    parts, h = [q, k, v], 1e-6
    for i, name in enumerate(("dq", "dk", "dv")):
        e = np.random.default_rng(i).standard_normal(parts[i].shape)
        up, down = list(parts), list(parts)
        up[i], down[i] = parts[i] + h * e, parts[i] - h * e
        d = sum((s * ref.attention(*x, lens, *how)["o"][0] * do).sum() for s, x in
                ((1, up), (-1, down))) / (2 * h)
        assert abs(d - (out[name][0] * e).sum()) < 1e-8 * np.abs(out[name][0] * e).sum() + 1e-9


def test_reference_steps_equal_causal_attention():
    # one position after another over a ring, against the window over all of them
    m, H, K, D, left, sinks = 30, 4, 2, 8, 6, 2
    q, k, v = data(m, H, K, D, 4)
    want = ref.attention(q, k, v, [m], left, 0, sinks, 0.3, False)["o"][0]
    kc, vc = (np.full((1, sinks + left + 1, K, D), np.nan) for _ in range(2))
    for i in range(m):
        o, _ = ref.step(q[i:i + 1], k[i:i + 1], v[i:i + 1], kc, vc, [i], left, sinks, 0.3, False)
        assert np.abs(o[0] - want[i]).max() < 1e-13


def test_reference_norm_rotate():
    rng = np.random.default_rng(5)
    n, H, D, sections = 6, 2, 12, [3, 2]
    x, w, dy = rng.standard_normal((n, H, D)), rng.standard_normal(D), rng.standard_normal((n, H, D))
    coords = rng.integers(-9, 9, (n, 3))
    freq = rng.random(6)
    y, _, dx, _, dw, _ = ref.norm_rotate(x, w, coords, freq, sections, 1e-3, False, dy)
    for t in range(n):  # term by term
        for g in range(H):
            u = w * x[t, g] / math.sqrt(sum(x[t, g] ** 2) / D + 1e-3)
            for j, a in enumerate([0, 0, 0, 1, 1, None]):
                z = complex(u[2 * j], u[2 * j + 1])
                if a is not None:
                    z *= complex(math.cos(coords[t, 1 + a] * freq[j]),
                                 math.sin(coords[t, 1 + a] * freq[j]))
                assert abs(complex(y[t, g, 2 * j], y[t, g, 2 * j + 1]) - z) < 1e-12
    h = 1e-6
    e, s = rng.standard_normal(x.shape), rng.standard_normal(D)

    def loss(a, b):
        return (ref.norm_rotate(a, b, coords, freq, sections, 1e-3, False)[0] * dy).sum()

    assert abs((loss(x + h * e, w) - loss(x - h * e, w)) / (2 * h) - (dx * e).sum()) < 1e-7
    assert abs((loss(x, w + h * s) - loss(x, w - h * s)) / (2 * h) - (dw * s).sum()) < 1e-7


@pytest.mark.parametrize("mistake", ["window", "sink", "group", "delta", "scale"])
def test_bounds_see_planted_mistakes(mistake):
    # the bounds that the kernels' tests use must not hide an off-by-one or a lost term
    lens, left, sinks = [40], 9, 2
    q, k, v = data(40, 4, 2, 16, 7)
    do = np.random.default_rng(8).standard_normal(q.shape)
    good = ref.attention(q, k, v, lens, left, 0, sinks, 0.25, True, do)
    if mistake == "window":
        bad = ref.attention(q, k, v, lens, left - 1, 0, sinks, 0.25, True, do)
    elif mistake == "sink":
        bad = ref.attention(q, k, v, lens, left, 0, sinks - 1, 0.25, True, do)
    elif mistake == "group":
        bad = ref.attention(q, k[:, ::-1], v[:, ::-1], lens, left, 0, sinks, 0.25, True, do)
    elif mistake == "scale":
        bad = ref.attention(q, k, v, lens, left, 0, sinks, 0.26, True, do)
    else:  # gradients that forget <do, o>
        see = ref.visible(40, left, 0, sinks)
        bad = {"dk": [np.zeros_like(k)], "dq": [np.zeros_like(q)]}
        for h in range(4):
            w = np.where(see, np.exp(0.25 * (q[:, h] @ k[:, h // 2].T)), 0)
            ds = 0.25 * w / w.sum(1, keepdims=True) * (do[:, h] @ v[:, h // 2].T)
            bad["dq"][0][:, h] = ds @ k[:, h // 2]
            bad["dk"][0][:, h // 2] += ds.T @ q[:, h]
    seen = [x for x in bad if (np.abs(bad[x][0] - good[x][0]) > good[x][1]).any()]
    assert ("dk" if mistake == "delta" else "o") in seen


class Heads(ctypes.Structure):
    _fields_ = [("p", P), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class Cache(ctypes.Structure):
    _fields_ = [("p", P), ("stream", ctypes.c_int64), ("row", ctypes.c_int64),
                ("head", ctypes.c_int64)]


def heads(p=4096, row=64, head=32):
    return ctypes.byref(Heads(p, row, head))


def message(lib):
    return lib.scn_last_error().decode()


def test_attention_refuses(lib):
    h = heads()

    def fwd(type=0, n=10, batch=1, ranges=P(4096), D=32, Hq=2, Hk=1, q=h, k=h, v=h, scale=1.0,
            sinks=0, o=h):
        return lib.scn_attn_fwd(type, n, batch, ranges, D, Hq, Hk, q, k, v, scale, -1, -1, sinks,
                                o, None, None)

    assert fwd(n=0) == 0  # nothing to do
    for kw, status, word in [
            (dict(type=2), 1, "type"), (dict(n=-1), 1, "size"), (dict(batch=0), 1, "size"),
            (dict(ranges=None), 1, "ranges"), (dict(Hq=3, Hk=2), 1, "multiple"),
            (dict(Hk=0), 1, "size"), (dict(scale=0.0), 1, "scale"), (dict(scale=-1.0), 1, "scale"),
            (dict(scale=float("nan")), 1, "scale"), (dict(scale=float("inf")), 1, "scale"),
            (dict(sinks=-1), 1, "sinks"), (dict(D=12), 5, "channels"), (dict(D=136), 5, "channels"),
            (dict(n=2 ** 30 + 1), 4, "2^30"), (dict(q=None), 1, "q is null"),
            (dict(k=heads(p=4100)), 1, "k must be"), (dict(v=heads(row=66)), 1, "v must be"),
            (dict(o=heads(head=33)), 1, "o must be"), (dict(q=heads(p=None)), 1, "q is null"),
            (dict(k=heads(row=-64)), 5, "rows"), (dict(k=heads(row=2 ** 22 + 8)), 5, "rows")]:
        assert fwd(**kw) == status, kw
        assert word in message(lib), (kw, message(lib))


def test_attention_backward_refuses(lib):
    h = heads()
    need = lib.scn_attn_bwd_workspace_bytes(100, 1, 32, 2, 1, -1, 0)
    assert need >= 100 * 2 * 4

    def bwd(lse=P(4096), ws=P(4096), ws_bytes=need, dq=h, sinks=0):
        return lib.scn_attn_bwd(0, 100, 1, P(4096), 32, 2, 1, h, h, h, h, lse, h, 1.0, -1, -1,
                                sinks, dq, h, h, ws, ws_bytes, None)

    assert bwd(lse=None) == 1 and bwd(dq=None) == 1 and bwd(sinks=-2) == 1
    assert bwd(ws=None) == 6 and bwd(ws_bytes=need - 1) == 6 and bwd(ws=P(4104)) == 6
    # a window with sinks takes the shares' room too, and no window none
    assert lib.scn_attn_bwd_workspace_bytes(100, 1, 32, 2, 1, 10, 3) > need
    assert lib.scn_attn_bwd_workspace_bytes(100, 1, 32, 2, 1, -1, 3) == need
    assert lib.scn_attn_bwd_workspace_bytes(-1, 1, 32, 2, 1, -1, 0) == 0


def test_step_refuses(lib):
    h, c = heads(), ctypes.byref(Cache(4096, 3200, 32, 32))

    def step(streams=2, cap=10, sinks=0, kc=c, length=P(4096), ws=None, ws_bytes=0, D=32):
        return lib.scn_attn_step(1, streams, cap, D, 1, 1, h, h, h, kc, c, length, 1.0, -1, sinks,
                                 h, ws, ws_bytes, None)

    assert step(streams=0) == 0
    assert step(streams=-1) == 1 and step(cap=4, sinks=4) == 1 and step(sinks=-1) == 1
    assert step(length=None) == 1 and step(kc=None) == 1 and step(D=20) == 5
    assert step(streams=65536) == 4 and step(cap=2 ** 30 + 1) == 4
    assert step(kc=ctypes.byref(Cache(4096, 3201, 32, 32))) == 1
    assert step(kc=ctypes.byref(Cache(4098, 3200, 32, 32))) == 1
    assert step(cap=2 ** 20) == 6  # long streams are split and need a workspace
    assert lib.scn_attn_step_workspace_bytes(1, 2, 2 ** 20, 32, 1, 1, -1, 0) > 0
    assert lib.scn_attn_step_workspace_bytes(1, 2, 100, 32, 1, 1, -1, 0) == 0
    assert lib.scn_attn_step_workspace_bytes(9, 2, 100, 32, 1, 1, -1, 0) == 0


def test_norm_rotate_refuses(lib):
    h = heads()

    def fwd(type=0, n=10, D=32, Hq=2, Hk=1, q=h, eps=1e-6, coords=P(4096), width=4, freq=P(4096),
            sections=(4, 4, 4), wq=None):
        sec = (ctypes.c_int32 * max(1, len(sections)))(*sections)
        return lib.scn_norm_rotate_fwd(type, n, D, Hq, Hk, q, h, wq, None, eps, coords, width, freq,
                                       sec, h, h, None)

    assert fwd(n=0) == 0
    for kw, status in [(dict(type=3), 1), (dict(n=-1), 1), (dict(Hq=0), 1), (dict(Hk=-1), 1),
                       (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(width=0), 1),
                       (dict(width=10, sections=(1,) * 9), 1), (dict(sections=(9, 4, 4)), 1),
                       (dict(sections=(-1, 4, 4)), 1), (dict(coords=None), 1), (dict(freq=None), 1),
                       (dict(q=None), 1), (dict(wq=P(4100)), 1), (dict(D=20), 5), (dict(D=256), 5),
                       (dict(n=2 ** 30 + 1), 4)]:
        assert fwd(**kw) == status, (kw, message(lib))
    need = lib.scn_norm_rotate_bwd_workspace_bytes(10, 32, 2, 1)
    assert need > 0
    sec = (ctypes.c_int32 * 3)(4, 4, 4)
    assert lib.scn_norm_rotate_bwd(0, 10, 32, 2, 1, h, h, None, None, 1e-6, P(4096), 4, P(4096), sec,
                                   h, h, h, h, P(4096), None, P(4096), need - 1, None) == 6
    assert lib.scn_site_ranges(None, 3, 4, 1, P(4096), None) == 1
    assert lib.scn_site_ranges(P(4096), 3, 0, 1, P(4096), None) == 1
    assert lib.scn_site_ranges(P(4096), 3, 4, 0, P(4096), None) == 1
    assert lib.scn_site_ranges(P(4096), 2 ** 31, 4, 1, P(4096), None) == 4
