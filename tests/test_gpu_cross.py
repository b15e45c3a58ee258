"""Cross attention on the GPU against the 64-bit reference: samples of any lengths on
both sides (none, one, a tile and one more), shared key heads, axes that are split over
blocks, strides, single rows of streams, values far from 1, other streams, graphs."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import block_reference as ref  # noqa: E402
from test_gpu_attention import TYPES, bounds, check, f64  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


def inputs(n, m, H, K, D, dtype, seed, fused=True):
    g = torch.Generator().manual_seed(seed)
    q = (1.5 * torch.randn(n, H, D, generator=g)).to(dtype).cuda()
    kv = torch.randn(m, 2 * K, D, generator=g).to(dtype).cuda()
    k, v = kv[:, :K], kv[:, K:]
    if not fused:
        k, v = k.contiguous(), v.contiguous()
    return q, k, v, torch.randn(n, H, D, generator=g).to(dtype).cuda()


# (rows of each sample, states of each, Hq, Hk, D)
CASES = [
    ([1], [1], 1, 1, 8),
    ([1, 1, 1], [5, 0, 33], 2, 1, 32),
    ([0, 5, 0, 64, 65], [7, 0, 0, 31, 129], 2, 2, 32),
    ([3, 127], [128, 257], 4, 1, 64),
    ([33, 200], [300, 2], 6, 2, 24),
    ([64], [700], 3, 1, 40),
    ([130, 20], [90, 191], 2, 1, 128),
    ([31, 257], [65, 40], 2, 2, 96),
    ([7], [2300], 4, 4, 64),               # keys split over blocks
    ([2, 0, 9], [4100, 50, 1030], 8, 2, 32),
    ([5], [3000], 2, 1, 112),
    ([2500, 1800], [3, 40], 2, 2, 32),     # queries split over blocks
    ([3000], [70], 4, 1, 64),
    ([2600], [33], 1, 1, 80),
    ([900, 700], [800, 1300], 2, 1, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_values_and_gradients(scn, case, dtype):
    ql, kl, H, K, D = CASES[case]
    q, k, v, do = inputs(sum(ql), sum(kl), H, K, D, TYPES[dtype], 70 + case, case % 2 == 0)
    how = dict(scale=0.3 if case % 3 == 0 else None)
    qr, kr = bounds(ql), bounds(kl)
    o, lse = scn.cross_attn_fwd(q, k, v, qr, kr, **how)
    d = scn.cross_attn_bwd(q, k, v, o, lse, do, qr, kr, **how)
    want = ref.cross(f64(q), f64(k), f64(v), ql, kl, how["scale"] or D ** -0.5, dtype == "bf16",
                     f64(do))
    empty = np.isinf(want["lse"][0])
    assert np.array_equal(np.isneginf(f64(lse)), empty)
    got = dict(o=o, **d)
    for name, t in got.items():
        check(name, t, *want[name])
    check("lse", torch.where(torch.isinf(lse), torch.zeros_like(lse), lse),
          np.where(empty, 0, want["lse"][0]), want["lse"][1])
    # the same bits again, on another stream too
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o2, lse2 = scn.cross_attn_fwd(q, k, v, qr, kr, **how)
        d2 = scn.cross_attn_bwd(q, k, v, o2, lse2, do, qr, kr, **how)
    s.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert all(torch.equal(d[x], d2[x]) for x in d)
