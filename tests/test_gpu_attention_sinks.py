"""Gradients of sinks whose far queries go to blocks of their own, in samples of more than
left + 256 rows: lengths on both sides of that, and short samples between long ones."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import attention_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LEFT = 30
EDGE = LEFT + 256


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


LENGTHS = {
    "edge": [EDGE, EDGE + 1, EDGE - 1, EDGE + 2, 0, EDGE + 1],
    "blocks": [511, 512, 513, 768, 769],
    "short between": [3, 700, 1, 0, 5, 2 * EDGE, 31, 32, 1030, 2],
    "one long": [7] * 150 + [1500] + [9] * 150,
    "short only": [40, 200, 286] * 5,
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("H,K,D,right,sinks", [(2, 1, 32, 0, 3), (2, 2, 64, 4, 40), (1, 1, 96, 0, 256),
                                               (2, 1, 128, 2, 33)])
def test_gradients(scn, dtype, lengths, H, K, D, right, sinks):
    lens = LENGTHS[lengths]
    n, t = sum(lens), TYPES[dtype]
    g = torch.Generator().manual_seed(len(lens) + D)
    q, k, v, do = (torch.randn(n, h, D, generator=g).to(t).cuda() for h in (H, K, K, H))
    r = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    how = dict(left=LEFT, right=right, sinks=sinks)
    o, lse = scn.attn_fwd(q, k, v, r, **how)
    # (room that holds NaN: nothing of it may be read before it is written)
    need = scn.lib().scn_attn_bwd_workspace_bytes(n, len(lens), D, H, K, LEFT, sinks)
    ws = torch.full((need // 4,), float("nan"), device="cuda").view(torch.uint8)
    d = scn.attn_bwd(q, k, v, o, lse, do, r, **how, ws=ws)
    want = ref.attention(*(x.double().cpu().numpy() for x in (q, k, v)), lens, LEFT, right, sinks,
                         D ** -0.5, dtype == "bf16", do.double().cpu().numpy())
    for name in ("dq", "dk", "dv"):
        x, (w, b) = d[name].double().cpu().numpy(), want[name]
        assert (np.abs(x - w) <= b).all(), name
