"""CPU checks of cross attention, block norms and clipping: the references' own pins
(differences, planted mistakes) and the calls' refusals."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest

import attention_reference as att
import block_reference as ref

P = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    import os

    from paper_1505_02890_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_1505_02890_amd.build import build
        build()
    return _lib.lib()


class Heads(ctypes.Structure):
    _fields_ = [("p", P), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class Rows(ctypes.Structure):
    _fields_ = [("p", P), ("row", ctypes.c_int64)]


class Tensor(ctypes.Structure):
    _fields_ = [("p", P), ("n", ctypes.c_int64), ("type", ctypes.c_int32)]


def heads(p=4096, row=64, head=32):
    return ctypes.byref(Heads(p, row, head))


def rows(p=4096, row=64):
    return ctypes.byref(Rows(p, row))


def message(lib):
    return lib.scn_last_error().decode()


# --------------------------------------------------------------------------
# references
# --------------------------------------------------------------------------

def data(n, m, H, K, D, seed):
    rng = np.random.default_rng(seed)
    return (rng.normal(size=(n, H, D)), rng.normal(size=(m, K, D)), rng.normal(size=(m, K, D)),
            rng.normal(size=(n, H, D)))


def test_cross_reference_is_attention_within_samples():
    # over its own rows, the other reference's values and bounds
    q, k, v, do = data(12, 12, 4, 2, 8, 0)
    a = att.attention(q, k, v, [5, 0, 7], None, None, 0, 0.3, True, do)
    b = ref.cross(q, k, v, [5, 0, 7], [5, 0, 7], 0.3, True, do)
    for x in a:
        assert np.allclose(a[x][0], b[x][0], rtol=1e-12, atol=1e-14), x
        assert np.allclose(a[x][1], b[x][1], rtol=0.2, atol=1e-9), x


def test_cross_reference_gradients_against_differences():
    ql, kl = [2, 0, 3, 1], [4, 2, 0, 1]
    q, k, v, do = data(6, 7, 2, 1, 4, 1)
    out = ref.cross(q, k, v, ql, kl, 0.4, False, do)
    assert np.all(out["o"][0][2:5] == 0) and np.all(np.isneginf(out["lse"][0][:, 2:5]))
    assert np.all(out["dk"][0][4:6] == 0) and np.all(out["dq"][0][2:5] == 0)
    for i, name in enumerate(("dq", "dk", "dv")):
        s = np.random.default_rng(5).normal(size=out[name][0].shape)

        def loss(e):
            t = [q, k, v]
            t[i] = t[i] + e * s
            return (ref.cross(*t, ql, kl, 0.4, False)["o"][0] * do).sum()

        num = (loss(1e-6) - loss(-1e-6)) / 2e-6
        assert abs(num - (out[name][0] * s).sum()) < 1e-7, name


@pytest.mark.parametrize("mistake", ["key", "group", "delta", "sample"])
def test_cross_bounds_see_planted_mistakes(mistake):
    q, k, v, do = data(40, 50, 4, 2, 16, 2)
    ql, kl = [15, 25], [30, 20]
    good = ref.cross(q, k, v, ql, kl, 0.25, True, do)
    if mistake == "key":  # the last key forgotten
        bad = ref.cross(q, k[:49], v[:49], ql, [30, 19], 0.25, True, do)
    elif mistake == "group":
        bad = ref.cross(q, k[:, ::-1], v[:, ::-1], ql, kl, 0.25, True, do)
    elif mistake == "sample":
        bad = ref.cross(q, k, v, [16, 24], kl, 0.25, True, do)
    else:
        half = ref.cross(q, k, v, ql, kl, 0.25, True, do * 0.97)
        bad = {"dq": half["dq"], "dk": half["dk"]}
    seen = [x for x in bad if x in good and bad[x][0].shape == good[x][0].shape and (
        np.abs(bad[x][0] - good[x][0]) > good[x][1]).any()]
    assert ("dq" if mistake == "delta" else "o") in seen


def block_data(n, C, seed):
    rng = np.random.default_rng(seed)
    return (*rng.normal(size=(3, n, C)), *(1 + 0.3 * rng.normal(size=(2, C))),
            *rng.normal(size=(2, n, C)))


def test_block_reference_gradients_against_differences():
    x, f, z, wf, wh, dy, dh = block_data(3, 7, 3)
    how = dict(alpha=0.7, eps=1e-3, res_bf16=False, bf16=False)
    g = ref.block(x, f, z, wf, wh, dy=dy, dh=dh, **how)
    t = dict(x=x, f=f, z=z, wf=wf, wh=wh)
    for name in t:
        s = np.random.default_rng(6).normal(size=t[name].shape)

        def loss(e):
            o = ref.block(**{**t, name: t[name] + e * s}, **how)
            return (o["y"][0] * dy).sum() + (o["h"][0] * dh).sum()

        num = (loss(1e-6) - loss(-1e-6)) / 2e-6
        assert abs(num - (g["d" + name][0] * s).sum()) < 1e-7, name


@pytest.mark.parametrize("mistake", ["eps", "mean", "gate", "alpha", "weight"])
def test_block_bounds_see_planted_mistakes(mistake):
    x, f, z, wf, wh, dy, dh = block_data(30, 75, 4)
    how = dict(alpha=0.9, eps=1e-6, res_bf16=True, bf16=True)
    good = ref.block(x, f, z, wf, wh, dy=dy, dh=dh, **how)
    t = dict(x=x, f=f, z=z, wf=wf, wh=wh, dy=dy, dh=dh)
    if mistake == "eps":
        bad = ref.block(**t, **{**how, "eps": 0.05})
    elif mistake == "alpha":
        bad = ref.block(**t, **{**how, "alpha": 0.92})
    elif mistake == "gate":
        bad = ref.block(**{**t, "z": z * 1.05}, **how)
    elif mistake == "weight":
        bad = ref.block(**{**t, "wf": np.roll(wf, 1)}, **how)
    else:  # the norm's gradient without its mean
        rf = 1 / np.sqrt((f * f).mean(1, keepdims=True) + 1e-6)
        bad = {"df": (good["dx"][0] / 0.9 * ref.sigmoid(z) * wf * rf, None)}
    assert any((np.abs(bad[n][0] - good[n][0]) > good[n][1]).any() for n in bad)


# --------------------------------------------------------------------------
# refusals
# --------------------------------------------------------------------------

def test_cross_attention_refuses(lib):
    h = heads()

    def fwd(type=0, nq=10, nk=20, batch=1, qr=P(4096), kr=P(4096), D=32, Hq=2, Hk=1, q=h, k=h, v=h,
            scale=1.0, o=h, ws=None, ws_bytes=0):
        return lib.scn_cross_attn_fwd(type, nq, nk, batch, qr, kr, D, Hq, Hk, q, k, v, scale, o,
                                      None, ws, ws_bytes, None)

    assert fwd(nq=0) == 0  # nothing to do
    for kw, status, word in [
            (dict(type=2), 1, "type"), (dict(nq=-1), 1, "size"), (dict(nk=-1), 1, "size"),
            (dict(batch=0), 1, "size"), (dict(qr=None), 1, "ranges"), (dict(kr=None), 1, "ranges"),
            (dict(Hq=3, Hk=2), 1, "multiple"), (dict(Hk=0), 1, "size"), (dict(scale=0.0), 1, "scale"),
            (dict(scale=float("nan")), 1, "scale"), (dict(D=12), 5, "channels"),
            (dict(D=136), 5, "channels"), (dict(nq=2 ** 30), 4, "2^30"),
            (dict(nk=2 ** 30 + 1), 4, "2^30"), (dict(q=None), 1, "q is null"),
            (dict(k=heads(p=4100)), 1, "k must be"), (dict(v=heads(row=66)), 1, "v must be"),
            (dict(o=heads(head=33)), 1, "o must be"), (dict(k=heads(p=None)), 1, "k is null"),
            (dict(k=heads(row=-64)), 5, "rows"), (dict(q=heads(row=2 ** 22 + 8)), 5, "rows"),
            (dict(nk=10 ** 6), 6, "workspace")]:
        assert fwd(**kw) == status, kw
        assert word in message(lib), (kw, message(lib))
    need = lib.scn_cross_attn_fwd_workspace_bytes(0, 10, 10 ** 6, 1, 32, 2, 1)
    assert need > 0 and fwd(nk=10 ** 6, ws=P(4096), ws_bytes=need - 1) == 6
    assert fwd(nk=10 ** 6, ws=P(4104), ws_bytes=need) == 6
    assert lib.scn_cross_attn_fwd_workspace_bytes(9, 10, 20, 1, 32, 2, 1) == 0
    assert lib.scn_cross_attn_fwd_workspace_bytes(0, 10, 20, 1, 32, 2, 1) == 0


def test_cross_attention_backward_refuses(lib):
    h = heads()
    need = lib.scn_cross_attn_bwd_workspace_bytes(0, 100, 50, 1, 32, 2, 1)
    assert need >= 3 * 100 * 2 * 4

    def bwd(lse=P(4096), ws=P(4096), ws_bytes=need, dq=h, dk=h, nq=100, nk=50):
        return lib.scn_cross_attn_bwd(0, nq, nk, 1, P(4096), P(4096), 32, 2, 1, h, h, h, h, lse, h,
                                      1.0, dq, dk, h, ws, ws_bytes, None)

    assert bwd(nq=0, nk=0) == 0
    assert bwd(lse=None) == 1 and bwd(dq=None) == 1 and bwd(dk=heads(p=4098)) == 1
    assert bwd(ws=None) == 6 and bwd(ws_bytes=need - 1) == 6 and bwd(ws=P(4104)) == 6
    assert lib.scn_cross_attn_bwd_workspace_bytes(0, -1, 50, 1, 32, 2, 1) == 0


@pytest.mark.parametrize("nq,nk,batch,H,K,D", [
    (1, 1 << 30, 1, 1, 1, 128), (1 << 20, 1 << 20, 1, 8, 8, 128), (1 << 20, 64, 1024, 16, 1, 64),
    (256, 1 << 24, 256, 64, 8, 128), (64, 1 << 22, 4, 4, 4, 64)])
@pytest.mark.parametrize("typ", [0, 1])
def test_workspaces_stay_small(lib, typ, nq, nk, batch, H, K, D):
    # parts are at most twice what fills the card four times, of 128 rows and 2 D + 1 floats,
    # or no larger than the results in fp32 times two; rows' statistics are three floats each
    blocks = 2 * 1024 * 2
    most = 4 * (blocks * 128 * (2 * D + 2) + 3 * (nq * H + 64))
    assert lib.scn_cross_attn_fwd_workspace_bytes(typ, nq, nk, batch, D, H, K) <= most
    assert lib.scn_cross_attn_bwd_workspace_bytes(typ, nq, nk, batch, D, H, K) <= most


def test_block_norm_refuses(lib):
    r = rows()

    def fwd(res=0, type=0, n=10, C=64, x=r, f=r, z=r, wf=None, wh=None, alpha=1.0, eps=1e-6, y=r,
            h=r):
        return lib.scn_block_norm_fwd(res, type, n, C, x, f, z, wf, wh, alpha, eps, y, h, None)

    assert fwd(n=0) == 0
    for kw, status, word in [
            (dict(res=2), 1, "type"), (dict(type=-1), 1, "type"), (dict(res=1), 5, "bf16"),
            (dict(n=-1), 1, "size"), (dict(C=0), 1, "size"), (dict(C=4097), 5, "channels"),
            (dict(eps=-1.0), 1, "eps"), (dict(eps=float("nan")), 1, "eps"),
            (dict(alpha=float("inf")), 1, "alpha"), (dict(n=2 ** 30 + 1), 4, "2^30"),
            (dict(x=None), 1, "x is null"), (dict(f=None), 1, "gate"),
            (dict(f=None, z=None, h=None), 1, "neither"), (dict(f=rows(p=None)), 1, "f is null"),
            (dict(x=rows(p=4098)), 1, "x is misaligned"), (dict(y=rows(row=-64)), 1, "y is"),
            (dict(wf=P(4097)), 1, "weights")]:
        assert fwd(**kw) == status, (kw, message(lib))
        assert word in message(lib), (kw, message(lib))
    need = lib.scn_block_norm_bwd_workspace_bytes(10, 64)
    assert need > 0 and lib.scn_block_norm_bwd_workspace_bytes(10, 5000) == 0

    def bwd(dx=r, df=r, dz=r, dwf=P(4096), ws=P(4096), ws_bytes=need, dh=r, f=r, z=r):
        return lib.scn_block_norm_bwd(0, 0, 10, 64, r, f, z, None, None, 1.0, 1e-6, None, dh, dx, df,
                                      dz, dwf, None, ws, ws_bytes, None)

    assert bwd(dx=None) == 1 and bwd(df=None) == 1 and bwd(dz=None) == 1
    assert bwd(f=None, z=None, dh=None) == 1
    assert bwd(ws=None) == 6 and bwd(ws_bytes=need - 1) == 6


def test_clip_refuses(lib):
    def clip(tensors, out=None, most=1.0, norm=P(4096), ws=P(4096), ws_bytes=1 << 20, count=None):
        a = (Tensor * max(1, len(tensors)))(*(Tensor(*t) for t in tensors))
        o = None if out is None else (P * len(out))(*out)
        return lib.scn_grad_clip(len(tensors) if count is None else count, a, o, most, norm, ws,
                                 ws_bytes, None)

    a, b = (1 << 20, 100000, 0), (1 << 24, 50, 1)
    for args, status, word in [
            (dict(tensors=[a], most=-1.0), 1, "largest norm"), (dict(tensors=[a], norm=None), 1, "norm"),
            (dict(tensors=[a], most=float("nan")), 1, "largest norm"),
            (dict(tensors=[a], count=-1), 1, "count"), (dict(tensors=[(4096, -1, 0)]), 1, "size"),
            (dict(tensors=[(4096, 1, 2)]), 1, "type"), (dict(tensors=[(None, 1, 0)]), 1, "null"),
            (dict(tensors=[(4098, 1, 0)]), 1, "misaligned"), (dict(tensors=[(4097, 1, 1)]), 1, "misaligned"),
            (dict(tensors=[a], out=[None]), 1, "null"), (dict(tensors=[(4096, 2 ** 40 + 1, 0)]), 4, "2^40"),
            (dict(tensors=[(4096, 2 ** 39, 0)] * 3), 4, "2^40"),
            (dict(tensors=[a], ws=None), 6, "workspace"), (dict(tensors=[a], ws_bytes=8), 6, "workspace"),
            (dict(tensors=[a, a]), 1, "overlap"), (dict(tensors=[a, ((1 << 20) + 399996, 4, 0)]), 1, "overlap"),
            (dict(tensors=[a, b], out=[1 << 28, (1 << 28) + 399998]), 1, "overlap"),
            (dict(tensors=[a, b], out=[1 << 28, (1 << 20) + 8]), 1, "overlap")]:
        assert clip(**args) == status, (args, message(lib))
        assert word in message(lib), (args, message(lib))
    assert lib.scn_grad_clip_workspace_bytes(5, 100) == 0
    assert lib.scn_grad_clip_workspace_bytes(1000, 100) > 0
    assert lib.scn_grad_clip_workspace_bytes(-1, 100) == 0
