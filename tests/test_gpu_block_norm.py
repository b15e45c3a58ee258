"""The norms around a block on the GPU against the 64-bit reference: types, channels that
fill lanes or do not, absent parts, strides and results in place, rows far from 1,
other streams, graphs, and gradients against differences."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import block_reference as ref  # noqa: E402
from test_gpu_attention import check, f64  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32,) * 2, "bf16": (torch.bfloat16,) * 2,
         "mixed": (torch.float32, torch.bfloat16)}


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


def inputs(n, C, kind, seed, gate=True):
    g = torch.Generator().manual_seed(seed)
    res, typ = TYPES[kind]
    r = lambda s, t: (s * torch.randn(n, C, generator=g)).to(t).cuda()  # noqa: E731
    x, f, z, dy, dh = r(2, res), r(0.5, typ), r(1, typ), r(1, res), r(1, typ)
    wf, wh = (1 + 0.3 * torch.randn(2, C, generator=g)).cuda()
    return x, f, z if gate else None, wf, wh, dy, dh


def opt(t):
    return None if t is None else f64(t)


def compare(scn, kind, x, f, z, wf, wh, dy, dh, alpha=0.875, eps=1e-6, y=None, h=None, d=None):
    res, typ = TYPES[kind]
    want = ref.block(f64(x), opt(f), opt(z), opt(wf), opt(wh), alpha, eps, res == torch.bfloat16,
                     typ == torch.bfloat16, opt(dy), opt(dh))
    if y is not None:
        check("y", y, *want["y"])
    if h is not None:
        check("h", h, *want["h"])
    for name, t in (d or {}).items():
        check(name, t, *want[name])


SIZES = [(1, 1), (3, 2), (5, 7), (17, 8), (1, 9), (33, 24), (70, 31), (64, 64), (257, 75), (5, 127),
         (40, 128), (19, 250), (9, 256), (130, 330), (7, 512), (6, 513), (3, 1000), (4, 1024),
         (5, 1031), (2, 2048), (3, 2055), (2, 4095), (2, 4096), (3001, 40)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,C", SIZES)
def test_values_and_gradients(scn, n, C, kind):
    t = inputs(n, C, kind, 100 * n + C, gate=(n + C) % 3 != 0)
    y, h = scn.block_norm_fwd(*t[:5], alpha=0.875)
    d = scn.block_norm_bwd(*t, alpha=0.875)
    compare(scn, kind, *t, y=y, h=h, d=d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2, h2 = scn.block_norm_fwd(*t[:5], alpha=0.875)
        d2 = scn.block_norm_bwd(*t, alpha=0.875)
    s.synchronize()
    assert torch.equal(y, y2) and torch.equal(h, h2) and all(torch.equal(d[k], d2[k]) for k in d)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("C", [64, 75, 600])
def test_absent_parts(scn, C, kind):
    x, f, z, wf, wh, dy, dh = inputs(41, C, kind, C)
    # a first block's norm; the last block's residual; no weights
    y, h = scn.block_norm_fwd(x, None, None, None, wh, need=("h",), out=(None, torch.empty_like(f)))
    assert y is None
    d = scn.block_norm_bwd(x, None, None, None, wh, dy, dh)
    assert set(d) == {"dx", "dwh"}
    compare(scn, kind, x, None, None, None, wh, dy, dh, alpha=1.0, h=h, d=d)
    y, h = scn.block_norm_fwd(x, f, z, wf, None, need=("y",))
    assert h is None
    d = scn.block_norm_bwd(x, f, z, wf, None, dy, None, need=("dwf",))
    assert set(d) == {"dx", "df", "dz", "dwf"}
    compare(scn, kind, x, f, z, wf, None, dy, None, alpha=1.0, y=y, d=d)
    y, h = scn.block_norm_fwd(x, f, None, None, None, alpha=-2.0, eps=0.1)
    d = scn.block_norm_bwd(x, f, None, None, None, None, dh, alpha=-2.0, eps=0.1, need=())
    assert set(d) == {"dx", "df"}
    compare(scn, kind, x, f, None, None, None, None, dh, alpha=-2.0, eps=0.1, y=y, h=h, d=d)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("C", [7, 96, 331, 1500])
def test_strides_and_places(scn, C, kind):
    t = inputs(29, C, kind, 7 + C)

    def wide(a, left, right):  # the same values, rows apart, from an odd element on
        w = torch.full((29, C + left + right), 5.0, dtype=a.dtype, device="cuda")
        w[:, left:left + C] = a
        return w, w[:, left:left + C]

    y, h = scn.block_norm_fwd(*t[:5])
    d = scn.block_norm_bwd(*t)
    (_, x), (_, f), (_, z), (_, dy), (_, dh) = (wide(a, i, 3 - i % 2) for i, a in enumerate(
        (t[0], t[1], t[2], t[5], t[6])))
    wy, oy = wide(y * 0, 1, 1)
    wh, oh = wide(h * 0, 3, 0)
    y2, h2 = scn.block_norm_fwd(x, f, z, t[3], t[4], out=(oy, oh))
    assert y2 is oy and torch.equal(y, y2) and torch.equal(h, h2)
    assert bool((wy[:, 0] == 5).all() and (wy[:, -1] == 5).all() and (wh[:, :3] == 5).all())
    d2 = scn.block_norm_bwd(x, f, z, t[3], t[4], dy, dh)
    assert all(torch.equal(d[k], d2[k]) for k in d)
    # in place: dx over dy, df over dh, dz over z; y over x, h over f
    x, f, z, dy, dh = (a.clone() for a in (t[0], t[1], t[2], t[5], t[6]))
    d3 = scn.block_norm_bwd(x, f, z, t[3], t[4], dy, dh, out=(dy, dh, z))
    assert d3["dx"] is dy and all(torch.equal(d[k], d3[k]) for k in d)
    z = t[2].clone()
    y3, h3 = scn.block_norm_fwd(x, f, z, t[3], t[4], out=(x, f))
    assert y3 is x and torch.equal(y, y3) and torch.equal(h, h3)
    # a gate that all rows share, read in place
    z1 = t[2][:1].expand(29, C)
    y4, _ = scn.block_norm_fwd(t[0], t[1], z1, t[3], t[4])
    y5, _ = scn.block_norm_fwd(t[0], t[1], z1.contiguous(), t[3], t[4])
    assert torch.equal(y4, y5)


@pytest.mark.parametrize("C", [8, 100, 520])
@pytest.mark.parametrize("size", [2.0 ** -75, 2.0 ** -55, 2.0 ** 55, 2.0 ** 62])
def test_rows_far_from_one(scn, C, size):
    # squares of such values leave fp32's range (or its best part); the norm does not depend on
    # the size where eps is 0, so the bounds stay those of rows of size 1
    x, f, z, wf, wh, dy, dh = inputs(23, C, "f32", C)
    f = f * size
    y, h = scn.block_norm_fwd(x, f, z, wf, wh, eps=0.0)
    d = scn.block_norm_bwd(x, f, z, wf, wh, dy, dh, eps=0.0)
    compare(scn, "f32", x, f, z, wf, wh, dy, dh, alpha=1.0, eps=0.0, y=y, h=h, d=d)
    # rows among others, and a residual of that size
    x = x.clone()
    x[::3] *= size
    y, h = scn.block_norm_fwd(x, f, z, wf, wh, eps=0.0)
    compare(scn, "f32", x, f, z, wf, wh, None, None, alpha=1.0, eps=0.0, y=y, h=h)


def test_gates_far_from_zero(scn):
    x, f, z, wf, wh, dy, dh = inputs(50, 64, "f32", 9)
    z = z * 25
    z[0, 0], z[0, 1], z[1, 0], z[1, 1] = 100, -100, float("inf"), -float("inf")
    y, h = scn.block_norm_fwd(x, f, z, wf, wh)
    d = scn.block_norm_bwd(x, f, z, wf, wh, dy, dh)
    compare(scn, "f32", x, f, z, wf, wh, dy, dh, alpha=1.0, y=y, h=h, d=d)


def test_special_rows_stay_alone(scn):
    # a row of NaN or infinities spoils its own results and the weights' sums, no other row
    x, f, z, wf, wh, dy, dh = inputs(30, 75, "f32", 4)
    y, h = scn.block_norm_fwd(x, f, z, wf, wh)
    f[4, 9], f[7, 0], x[11, 74] = float("nan"), float("inf"), -float("inf")
    y2, h2 = scn.block_norm_fwd(x, f, z, wf, wh)
    others = [i for i in range(30) if i not in (4, 7, 11)]
    assert torch.equal(y[others], y2[others]) and torch.equal(h[others], h2[others])
    assert bool(y2[4].isnan().all()) and bool(h2[7].isnan().any()) and bool(h2[11].isnan().any())
    f.zero_()  # n(0) is 0 with eps, and nothing without
    y, h = scn.block_norm_fwd(dy, f, z, wf, wh)
    assert torch.equal(y, dy)
    y, h = scn.block_norm_fwd(dy, f, z, wf, wh, eps=0.0)
    assert bool(y.isnan().all())


def test_no_rows(scn):
    e = torch.empty(0, 24, device="cuda")
    w = torch.ones(24, device="cuda")
    y, h = scn.block_norm_fwd(e, e, None, w, w)
    assert y.shape == h.shape == (0, 24)
    d = scn.block_norm_bwd(e, e, e, w, w, e, e)
    assert float(d["dwf"].abs().sum()) == float(d["dwh"].abs().sum()) == 0


def test_gradients_against_differences(scn):
    # central differences of the 64-bit reference
    x, f, z, wf, wh, dy, dh = (f64(t) for t in inputs(4, 11, "f32", 12))

    def loss(**k):
        o = ref.block(**{**dict(x=x, f=f, z=z, wf=wf, wh=wh, alpha=0.7, eps=1e-3, res_bf16=False,
                                bf16=False), **k})
        return (o["y"][0] * dy).sum() + (o["h"][0] * dh).sum()

    t = {n: torch.tensor(a, dtype=torch.float32).cuda() for n, a in dict(
        x=x, f=f, z=z, wf=wf, wh=wh, dy=dy, dh=dh).items()}
    d = scn.block_norm_bwd(**t, alpha=0.7, eps=1e-3)
    for name, a in dict(x=x, f=f, z=z, wf=wf, wh=wh).items():
        num = np.zeros_like(a)
        for i in np.ndindex(a.shape):
            s = np.zeros_like(a)
            s[i] = 1e-5
            num[i] = (loss(**{name: a + s}) - loss(**{name: a - s})) / 2e-5
        # differences are off by 1e-10 / 2e-5 of rounding and 1e-10 of curvature; the kernel by
        # some hundred units of fp32
        assert np.abs(f64(d["d" + name]) - num).max() <= 2e-5 * max(1, np.abs(num).max()), name


@pytest.mark.parametrize("C", [64, 330, 1031])
def test_graph(scn, C):
    t = inputs(300, C, "mixed", C)
    scn.block_norm_fwd(*t[:5])
    scn.block_norm_bwd(*t)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, h = scn.block_norm_fwd(*t[:5])
        d = scn.block_norm_bwd(*t)
    for seed in range(3):
        for a, b in zip(t, inputs(300, C, "mixed", seed)):
            a.copy_(b)
        want = scn.block_norm_fwd(*t[:5]), scn.block_norm_bwd(*t)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0][0]) and torch.equal(h, want[0][1])
        assert all(torch.equal(d[k], want[1][k]) for k in d)
