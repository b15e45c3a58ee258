"""Norm and rotation of rows far from 1: the gradients' terms lie between 1 / |x| and 1 in
size, however small or large x is."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import attention_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("power,eps", [(-55, 0.0), (-46, 0.0), (-40, 1e-30), (-20, 1e-6), (20, 1e-6),
                                       (40, 1e-6), (46, 1e-6), (55, 0.0)])
@pytest.mark.parametrize("n,H,D", [(70, 3, 32), (9000, 8, 64)])
def test_norm_rotate(scn, dtype, power, eps, n, H, D):
    g = torch.Generator().manual_seed(5)
    q = (torch.randn(n, H, D, generator=g) * 2.0 ** power).to(dtype).cuda()
    dy = torch.randn(n, H, D, generator=g).to(dtype).cuda()
    w = (1 + 0.3 * torch.randn(D, generator=g)).cuda()
    coords = torch.randint(0, 64, (n, 4), generator=g).to(torch.int32).cuda()
    sections = [D // 8] * 3
    freq = scn.rotation_freqs(D, sections)
    y, _ = scn.norm_rotate_fwd(q, None, w, None, coords, freq, sections, eps=eps)
    d = scn.norm_rotate_bwd(q, None, w, None, coords, freq, sections, dy, None, eps=eps)
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    want = ref.norm_rotate(f64(q), f64(w), coords.cpu().numpy(), f64(freq), sections, eps,
                           dtype == torch.bfloat16, f64(dy))
    for name, got, (value, bound) in zip(("y", "dq", "dw"), (y, d["dq"], d["dwq"]),
                                         (want[:2], want[2:4], want[4:])):
        # gradients of x ~ 2^power are of size 2^-power
        off = np.abs(f64(got) - value)
        assert np.isfinite(f64(got)).all() and (off <= bound).all(), name
