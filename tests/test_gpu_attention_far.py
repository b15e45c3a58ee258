"""Rows and cache slots whose offsets pass 32 bits."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import attention_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    if torch.cuda.get_device_properties(0).total_memory < 150 << 30:
        pytest.skip("needs some 40 GB of device memory")
    return m


def f64(t):
    torch.cuda.synchronize()
    return t.detach().double().cpu().numpy()


def check(name, got, want, tol):
    assert (np.abs(f64(got) - want) <= tol).all(), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart(scn, dtype):
    # rows 2^22 elements apart, the most that a call takes: the last ones lie 2^32 elements
    # and more from the first
    lens, H, K, D, row = [700, 1, 400], 2, 1, 32, 1 << 22
    n, t = sum(lens), TYPES[dtype]
    g = torch.Generator().manual_seed(1)
    big = torch.empty(n * row, dtype=t, device="cuda")
    rows = big.view(n, row)[:, :(4 * H + 4 * K) * D].unflatten(1, (4 * H + 4 * K, D))
    rows.copy_(torch.randn(n, 4 * H + 4 * K, D, generator=g))
    parts = torch.split(rows, [H, K, K, H, H, H, K, K], 1)
    q, k, v, do, o, dq, dk, dv = parts
    assert q.stride(0) == row and (n - 1) * row >= 2 ** 32
    how = dict(left=100, right=3, sinks=2)
    r = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    want = ref.attention(f64(q), f64(k), f64(v), lens, 100, 3, 2, D ** -0.5, dtype == "bf16",
                         f64(do))
    _, lse = scn.attn_fwd(q, k, v, r, **how, out=o)
    d = scn.attn_bwd(q, k, v, o, lse, do, r, **how, out=(dq, dk, dv))
    for name, got in dict(o=o, lse=lse, **d).items():
        check(name, got, *want[name])
    coords = torch.randint(0, 64, (n, 3), generator=g).to(torch.int32).cuda()
    sections = [8, 8]
    freq = scn.rotation_freqs(D, sections)
    y, _ = scn.norm_rotate_fwd(q, None, None, None, coords, freq, sections, out=(o, None))
    d = scn.norm_rotate_bwd(q, None, None, None, coords, freq, sections, do, None, out=(dq, None))
    ry, ty, dx, tx, dw, tw = ref.norm_rotate(f64(q), None, coords.cpu().numpy(), f64(freq), sections,
                                             1e-6, dtype == "bf16", f64(do))
    check("y", y, ry, ty)
    check("dq", d["dq"], dx, tx)
    check("dw", d["dwq"], dw, tw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left,length", [(63, 1_100_000), (None, 1500), (700, 2_300_017)])
def test_long_caches(scn, dtype, left, length):
    # 16 heads of 128 channels: slots from 2^21 on lie past 2^32 elements
    H, K, D, cap, sinks = 32, 16, 128, (1 << 21) + 70_000, 3
    t = TYPES[dtype]
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(1, h, D, generator=g).to(t).cuda() for h in (H, K, K))
    kc, vc = (torch.empty(1, cap, K, D, dtype=t, device="cuda") for _ in range(2))
    ring = cap - sinks
    reach = ring - 1 if left is None else left
    seen = list(range(sinks)) + [sinks + (j - sinks) % ring
                                 for j in range(max(sinks, length - reach), length)]
    at = torch.tensor(seen, device="cuda")
    for c in (kc, vc):
        c[0, at] = torch.randn(len(seen), K, D, generator=g).to(t).cuda()
    keys = np.concatenate([f64(kc[0, at]), f64(k)]), np.concatenate([f64(vc[0, at]), f64(v)])
    o = scn.attn_step(q, k, v, kc, vc, torch.tensor([length], dtype=torch.int32, device="cuda"),
                      left=left, sinks=sinks)
    # the same keys in a small cache
    m = len(seen)
    small = [np.concatenate([x[:m], np.zeros((1, K, D))])[None] for x in keys]
    want, tol = ref.step(f64(q), f64(k), f64(v), *small, [m], None, 0, D ** -0.5, dtype == "bf16")
    check("o", o, want, tol)
    now = sinks + (length - sinks) % ring
    assert torch.equal(kc[0, now], k[0]) and torch.equal(vc[0, now], v[0])
