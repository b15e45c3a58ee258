"""A first block's norm in place: y over x without a block's result, where the last lane
of a row reads and writes channels that a lane of another wave writes too (rows of 512 m
+ 1 to 7 channels)."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from test_gpu_block_norm import TYPES, compare, inputs  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("C", [75, 505, 512, 513, 519, 520, 1031, 2049, 3591])
def test_y_over_x_without_f(scn, C, kind):
    x, f, _, _, wh, dy, dh = inputs(700, C, kind, C)
    y, h = scn.block_norm_fwd(x, None, None, None, wh, alpha=0.875, out=(None, torch.empty_like(f)))
    compare(scn, kind, x, None, None, None, wh, None, None, y=y, h=h)
    for _ in range(3):
        place, h2 = x.clone(), torch.empty_like(f)
        y2, _ = scn.block_norm_fwd(place, None, None, None, wh, alpha=0.875, out=(place, h2))
        assert y2 is place and torch.equal(y, y2) and torch.equal(h, h2)
    # backward: dx over dy
    d = scn.block_norm_bwd(x, None, None, None, wh, dy, dh, alpha=0.875)
    place = dy.clone()
    d2 = scn.block_norm_bwd(x, None, None, None, wh, place, dh, alpha=0.875, out=(place, None, None))
    assert d2["dx"] is place and all(torch.equal(d[k], d2[k]) for k in d)
