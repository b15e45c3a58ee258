"""The block of ``cross.py`` on rows and states of any number of channels: values against 64
bits, gradients against differences, streams."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import bounds, f64  # noqa: E402
from test_gpu_cross_block import forward64  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("channels,states,heads,kv,dim", [
    (50, 16, 4, 2, 16), (75, 9, 2, 1, 8), (7, 5, 1, 1, 8), (33, 64, 2, 2, 40), (24, 31, 2, 1, 32)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_any_channels(scn, dtype, channels, states, heads, kv, dim):
    # bounds as in test_gpu_cross_block: fp32 some 1e-6 of values up to 5, with a factor of ten;
    # bf16 a rounding of q, k, v, o and the weights, some 2^-8 each of values up to 5
    from paper_1505_02890_amd.cross import CrossBlock, _line
    qlens, klens = [5, 0, 9, 3], [7, 4, 0, 40]
    block = CrossBlock(channels, states, heads, kv, dim, alpha=0.9, dtype=dtype, seed=3)
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    x, m = r(17, channels), r(51, states)
    sites, ms, qr, kr = _line(17), _line(51), bounds(qlens), bounds(klens)
    h = block.enter(x)
    y, hn, saved = block.forward(sites, qr, x, h, ms, kr, m)
    params = {k: f64(w) for k, w in block.params.items()}
    X, Hh, M = f64(x), f64(h), f64(m)
    wy, wh = forward64(block, params, qlens, klens, X, Hh, M)
    lim = 2e-5 if dtype == torch.float32 else 0.15
    assert np.abs(f64(y) - wy).max() < lim and np.abs(f64(hn) - wh).max() < lim
    dy, dh = r(*y.shape), r(*y.shape)
    dx, dhin, dm, grads = block.backward(saved, dy, dh)
    if dtype == torch.float32:
        def loss(p=params, X=X, Hh=Hh, M=M):
            a, b = forward64(block, p, qlens, klens, X, Hh, M)
            return (a * f64(dy)).sum() + (b * f64(dh)).sum()

        rng = np.random.default_rng(0)
        for name, got in dict(grads, X=dx, Hh=dhin, M=dm).items():
            base = {"X": X, "Hh": Hh, "M": M}.get(name, params.get(name))
            s = rng.normal(size=base.shape)
            at = lambda e: loss(p={**params, name: base + e * s}) if name in params else loss(  # noqa: E731
                **{name: base + e * s})
            num = (at(1e-5) - at(-1e-5)) / 2e-5
            parts = f64(got).reshape(base.shape) * s
            assert abs(parts.sum() - num) < 1e-5 * (np.abs(parts).sum() + 1), name
    st = block.open(ms, kr, m)
    at = torch.minimum(qr[:-1].long() + 1, qr[1:].long() - 1).clamp(min=0)
    some = [0, 2, 3]  # (streams whose stroke has rows)
    a, b = block.step(st, x[at], h[at])
    lim = 1e-4 if dtype == torch.float32 else 0.1
    assert float((a - y[at])[some].abs().max()) < lim and float((b - hn[at])[some].abs().max()) < lim
