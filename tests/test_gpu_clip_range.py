"""Clipping at the ends of fp32's range: norms on both sides of its largest number, scales
below its smallest.  In one launch and in two kernels."""
from __future__ import annotations

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import f64  # noqa: E402
from test_gpu_clip import B, F, check, make  # noqa: E402

pytestmark = pytest.mark.gpu

FEW, MANY = [1000, 3001], [60000, 30001]  # elements of a small call, and past it
LARGEST = float(np.finfo(np.float32).max)


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("kinds", [[F], [B], [F, B]], ids=["f32", "bf16", "both"])
@pytest.mark.parametrize("sizes", [FEW, MANY], ids=["few", "many"])
def test_norms_around_the_largest_number(scn, sizes, kinds):
    # all elements of one size: the norm is that size times the root of their number
    root = math.sqrt(sum(sizes))
    for share in (0.98, 1.02):
        grads = [torch.full((n,), share * LARGEST / root, dtype=kinds[i % len(kinds)], device="cuda")
                 for i, n in enumerate(sizes)]
        exact = [f64(t) for t in grads]
        norm = math.sqrt(sum(float((g * g).sum()) for g in exact))
        out = [torch.zeros_like(t) for t in grads]
        if share < 1:
            assert norm < LARGEST
            check(scn.clip_grads(grads, norm / 2, out=out), out, exact, norm / 2)
            check(scn.clip_grads(grads, norm / 2), grads, exact, norm / 2)
        else:
            assert norm > LARGEST
            for place in (out, grads):
                got = scn.clip_grads(grads, norm / 2, out=None if place is grads else out)
                assert math.isinf(float(got))
                assert all(np.array_equal(f64(t), g) for t, g in zip(place, exact))


def test_two_numbers_near_the_largest(scn):
    for dtype in (F, B):
        t = torch.tensor([3e38, 3e38], dtype=dtype, device="cuda")
        keep = t.clone()
        assert math.isinf(float(scn.clip_grads([t], 1.0)))
        assert torch.equal(t, keep)


@pytest.mark.parametrize("kinds", [[F], [B], [F, B]], ids=["f32", "bf16", "both"])
@pytest.mark.parametrize("sizes", [FEW, MANY], ids=["few", "many"])
@pytest.mark.parametrize("most", [1e-3, 1e-6, 1e-8])
def test_scales_below_the_smallest_number(scn, sizes, kinds, most):
    # a norm of 1e37: the scale has few bits or none in fp32, the results are ordinary numbers
    grads = make(sizes, kinds, 3, std=1e37 / math.sqrt(sum(sizes)))
    exact = [f64(t) for t in grads]
    out = [torch.zeros_like(t) for t in grads]
    check(scn.clip_grads(grads, most, out=out), out, exact, most)
    assert all(float(t.abs().max()) > 0 for t in out)
    check(scn.clip_grads(grads, most), grads, exact, most)
