"""Cross attention of few rows of 40, 48 and 56 channels, and of heads that lie outside their
rows ([heads, rows, channels], as other code keeps them): values and gradients against the
64-bit reference, the bits of dense calls in other layouts with rows of no sample in front,
streams of a layer with such heads."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import TYPES, bounds  # noqa: E402
from test_gpu_cross import inputs  # noqa: E402
from test_gpu_cross_shapes import LENS, compare  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


# few rows: one, some on states in parts, tiles that end inside and at 32 rows, states of any
# number around a tile's
FEW = {
    "one": LENS["one"],
    "thin": LENS["thin"],
    "streams": ([1] * 40, [(97 * i) % 700 for i in range(40)]),
    "far": ([2], [40000]),
    "tile": ([4, 8, 7], [31, 32, 33]),
    "none": ([3, 2], [0, 0]),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,K", [(1, 1), (4, 2), (6, 2), (4, 4)])
@pytest.mark.parametrize("D", [40, 48, 56])
@pytest.mark.parametrize("which", list(FEW))
def test_few_rows(scn, which, D, H, K, dtype):
    ql, kl = FEW[which]
    q, k, v, do = inputs(sum(ql), sum(kl), H, K, D, TYPES[dtype], D + H)
    if sum(kl) == 0:
        qr, kr = bounds(ql), bounds(kl)
        o, lse = scn.cross_attn_fwd(q, k, v, qr, kr)
        d = scn.cross_attn_bwd(q, k, v, o, lse, do, qr, kr)
        assert not o.any() and not d["dq"].any() and bool(torch.isneginf(lse).all())
        return
    compare(scn, q, k, v, do, ql, kl, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,K,D", [(4, 2, 32), (4, 4, 56), (6, 2, 64), (4, 1, 96), (2, 2, 128)])
@pytest.mark.parametrize("which", ["thin", "one", "some", "rows", "text2"])
@pytest.mark.parametrize("front", [0, 1, 200])
def test_heads_outside_their_rows(scn, front, which, H, K, D, dtype):
    ql, kl = LENS[which]
    n, m = sum(ql), sum(kl)
    q, k, v, do = inputs(n, m, H, K, D, TYPES[dtype], 3)
    qr, kr = bounds(ql), bounds(kl)
    # (the plan goes by the rows: those of no sample count in both calls)
    pad = lambda t, fill: torch.cat([torch.full((front, *t.shape[1:]), fill, dtype=t.dtype,  # noqa: E731
                                                device="cuda"), t])
    q, k, v, do = (pad(t, float("nan")) for t in (q, k, v, do))
    qr, kr = qr + front, kr + front
    o, lse = scn.cross_attn_fwd(q, k, v, qr, kr)
    d = scn.cross_attn_bwd(q, k, v, o, lse, do, qr, kr)

    def heads_first(t):
        return t.permute(1, 0, 2).contiguous().permute(1, 0, 2)

    outs = [heads_first(torch.full((r, h, D), 7.0, dtype=TYPES[dtype], device="cuda"))
            for r, h in ((n + front, H), (n + front, H), (m + front, K), (m + front, K))]
    q2, k2, v2, do2 = (heads_first(t) for t in (q, k, v, do))
    o2, lse2 = scn.cross_attn_fwd(q2, k2, v2, qr, kr, out=outs[0])
    d2 = scn.cross_attn_bwd(q2, k2, v2, o2, lse2, do2, qr, kr, out=tuple(outs[1:]))
    assert torch.equal(o2[front:], o[front:]) and torch.equal(lse2[:, front:], lse[:, front:])
    assert all(torch.equal(d2[x][front:], d[x][front:]) for x in d)
    assert all(bool((t[:front] == 7.0).all()) for t in outs)


@pytest.mark.parametrize("dim", [40, 56])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_streams_of_a_layer(scn, dtype, dim):
    # bounds as in test_gpu_cross_block's streams
    from paper_1505_02890_amd.cross import CrossBlock, _line
    qlens, klens = [6, 4, 9], [700, 0, 33]
    block = CrossBlock(24, 16, heads=4, kv=2, dim=dim, dtype=dtype, seed=3)
    g = torch.Generator().manual_seed(3)
    x, m = (torch.randn(*s, generator=g).cuda() for s in ((19, 24), (733, 16)))
    h = block.enter(x)
    qr, kr = bounds(qlens), bounds(klens)
    ms = _line(733)
    y, hn, saved = block.forward(_line(19), qr, x, h, ms, kr, m)
    grads = block.backward(saved, torch.ones_like(y), None)[3]
    assert all(bool(torch.isfinite(t).all()) for t in grads.values())
    st = block.open(ms, kr, m)
    first = qr[:-1].long()
    for i in range(4):
        a, b = block.step(st, x[first + i], h[first + i])
        lim = 1e-4 if dtype == torch.float32 else 0.1
        assert float((a - y[first + i]).abs().max()) < lim
        assert float((b - hn[first + i]).abs().max()) < lim
