"""Attention's gradients in bf16 where few of many keys hold a row's weight: dP - <do, o>
nearly cancels there, which the rounding of o to bf16 must not reach."""
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


# As where rows see few keys: two independent roundings to bf16, of dS and of the result,
# each of at most 2^-8 / sqrt(3) in the root mean square; the sums are in fp32.
FROBENIUS = 2 ** 0.5 * 2.0 ** -8 / 3 ** 0.5


@pytest.mark.parametrize("D", [32, 64, 96, 104, 128])
@pytest.mark.parametrize("gain", [1.5, 4.0, 8.0, 16.0])
@pytest.mark.parametrize("lens,left,right", [
    ([512, 300], None, None), ([700], None, 0), ([1100], 255, 64), ([1024], None, None)])
def test_peaked_rows(scn, D, gain, lens, left, right):
    H, K, n = 4, 2, sum(lens)
    g = torch.Generator().manual_seed(int(gain * 10) + D)
    q, k, v, do = (torch.randn(n, h, D, generator=g) for h in (H, K, K, H))
    q, k, v, do = (t.to(torch.bfloat16).cuda() for t in (q * gain, k, v, do))
    ranges = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    o, lse = scn.attn_fwd(q, k, v, ranges, left=left, right=right)
    got = scn.attn_bwd(q, k, v, o, lse, do, ranges, left=left, right=right)
    want = ref.attention(*(t.double().cpu().numpy() for t in (q, k, v)), lens, left, right, 0,
                         D ** -0.5, True, do.double().cpu().numpy())
    for name in ("dq", "dk", "dv"):
        x, w = got[name].double().cpu().numpy(), want[name][0]
        off = np.linalg.norm(x - w) / np.linalg.norm(w)
        assert off <= FROBENIUS, (name, off)
