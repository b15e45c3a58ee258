"""The attention layer: sites of no sample, and streams of layers that are not causal."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


def layer_of(dtype, **kw):
    from paper_1505_02890_amd.attention import SiteAttention
    return SiteAttention(32, heads=4, kv=2, dim=16, dtype=dtype, seed=2, **kw)


def litter(n):
    """Leaves NaN in the memory that the next tensors of a layer get."""
    held = [torch.full((n, c), float("nan"), device="cuda", dtype=t)
            for c in (16, 32, 64, 128) for t in (torch.float32, torch.bfloat16) for _ in range(4)]
    torch.cuda.synchronize()
    del held


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sites_of_no_sample(scn, dtype):
    # the last sample's sites are past the ranges: they pass unchanged, and teach nothing
    from paper_1505_02890_amd.attention import _strokes
    lens = [70, 45, 80]
    inside = sum(lens[:2])
    layer = layer_of(dtype, left=20, right=0, sinks=2)
    coords, sites = _strokes(lens, 40, 5)
    few, few_sites = _strokes(lens[:2], 40, 5)
    n = len(coords)
    g = torch.Generator().manual_seed(3)
    x, dy = (torch.randn(n, 32, generator=g).cuda() for _ in range(2))
    assert torch.equal(few, coords[:inside])
    ranges = scn.site_ranges(coords, 2)
    litter(n)
    y, saved = layer.forward(sites, coords, ranges, x)
    litter(n)
    dx, grads = layer.backward(saved, dy)
    want, kept = layer.forward(few_sites, few, scn.site_ranges(few, 2), x[:inside].contiguous())
    wdx, wgrads = layer.backward(kept, dy[:inside].contiguous())
    assert torch.equal(y[inside:], x[inside:]) and torch.equal(dx[inside:], dy[inside:])
    assert torch.allclose(y[:inside], want, rtol=0, atol=1e-5)
    assert torch.allclose(dx[:inside], wdx, rtol=0, atol=1e-5)
    for name in grads:  # sums over other numbers of rows, in other orders
        assert torch.allclose(grads[name], wgrads[name], rtol=1e-4, atol=1e-4), name


@pytest.mark.parametrize("right", [None, 1, 40])
def test_streams_need_a_causal_layer(scn, right):
    # a stream's newest point cannot see the ones after it
    with pytest.raises(ValueError, match="causal"):
        layer_of(torch.float32, left=20, right=right).open(2, 30)


@pytest.mark.parametrize("capacity", [0, 3, 4])
def test_streams_need_room_past_the_sinks(scn, capacity):
    with pytest.raises(ValueError, match="capacity"):
        layer_of(torch.float32, left=20, right=0, sinks=4).open(2, capacity)
