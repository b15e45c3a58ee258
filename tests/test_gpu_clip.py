"""Clipping by the global norm on the GPU against 64 bits: sizes around a block's
share and its vectors, both types in one call, more tensors than a launch takes, places
that begin anywhere, norms that are not finite, graphs."""
from __future__ import annotations

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import f64  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


def make(sizes, kinds, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(std * torch.randn(n, generator=g)).to(kinds[i % len(kinds)]).cuda()
            for i, n in enumerate(sizes)]


def check(norm, out, grads, most):
    """grads: float64 arrays.  The sum of squares is in 64 bits and rounds once to fp32;
    the scale too, for bf16 (a float and a product of floats more), and results round once."""
    want = math.sqrt(sum(float((g * g).sum()) for g in grads))
    assert abs(float(norm) - want) <= 2.0 ** -23.9 * want
    by = most / want if want > most else 1.0
    for t, g in zip(out, grads):
        u = 2.0 ** -8 if t.dtype == torch.bfloat16 else 2.0 ** -24
        bound = (1.01 * u + (2.0 ** -23 if t.dtype == torch.bfloat16 else 0)) * np.abs(g * by) + (
            0 if by == 1 else 1e-40)
        if by == 1:
            bound = 0 * bound
        assert np.all(np.abs(f64(t) - g * by) <= bound)


F, B = torch.float32, torch.bfloat16
SIZES = [[1], [3, 0, 5], [4, 8, 7, 9], [8191, 8192, 8193], [16385, 1, 33], [100000, 20001],
         [17] * 300, [5000] * 129, [3000000, 2, 999983]]


@pytest.mark.parametrize("kinds", [[F], [B], [F, B]], ids=["f32", "bf16", "both"])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_norm_and_clipping(scn, case, kinds):
    grads = make(SIZES[case], kinds, case)
    exact = [f64(t) for t in grads]
    norm = math.sqrt(sum(float((g * g).sum()) for g in exact))
    out = [torch.full_like(t, 9.0) for t in grads]
    for most in (norm / 3, norm * 3, math.inf, 0.0):
        check(scn.clip_grads(grads, most, out=out), out, exact, most)
        assert all(np.array_equal(f64(t), g) for t, g in zip(grads, exact))
    check(scn.clip_grads(grads, 2 * norm), grads, exact, 2 * norm)
    check(scn.clip_grads(grads, norm / 7), grads, exact, norm / 7)
    # the same bits on another stream
    again = make(SIZES[case], kinds, case)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        scn.clip_grads(again, norm / 7)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


def test_places_that_begin_anywhere(scn):
    g = torch.Generator().manual_seed(1)
    for dtype in (F, B):
        flat = torch.randn(60000, generator=g).to(dtype).cuda()
        keep = flat.clone()
        cut = [0, 1, 8, 17, 8300, 8301, 20003, 59999]
        parts = [flat[a + (i % 2):b] for i, (a, b) in enumerate(zip(cut, cut[1:]))]
        exact = [f64(t) for t in parts]
        check(scn.clip_grads(parts, 1.5), parts, exact, 1.5)
        inside = torch.zeros(60000, dtype=torch.bool, device="cuda")
        for i, (a, b) in enumerate(zip(cut, cut[1:])):
            inside[a + (i % 2):b] = True
        assert torch.equal(flat[~inside], keep[~inside])


def test_far_from_one(scn):
    # squares leave fp32's range, the norm and the results do not
    for size in (1e-30, 1e-22, 1e25, 1e36):
        grads = make([1000, 3001], [F, B], 5, std=size)
        exact = [f64(t) for t in grads]
        norm = math.sqrt(sum(float((g * g).sum()) for g in exact))
        check(scn.clip_grads(grads, norm / 2), grads, exact, norm / 2)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_norms_that_are_not_finite(scn, bad):
    grads = make([900, 12001], [F, B], 6)
    grads[1][7] = bad
    keep = [t.clone() for t in grads]
    norm = scn.clip_grads(grads, 0.5)
    assert not math.isfinite(float(norm)) and math.isnan(float(norm)) == math.isnan(bad)
    assert all(torch.equal(a[a == a], b[b == b]) for a, b in zip(grads, keep))
    out = [torch.zeros_like(t) for t in grads]
    scn.clip_grads(grads, 0.5, out=out)
    assert all(torch.equal(a[a == a], b[b == b]) for a, b in zip(out, keep))


def test_nothing_to_clip(scn):
    assert float(scn.clip_grads([], 1.0)) == 0
    e = [torch.empty(0, device="cuda"), torch.empty(3, 0, dtype=B, device="cuda")]
    assert float(scn.clip_grads(e, 1.0)) == 0
    z = [torch.zeros(100, device="cuda")]
    assert float(scn.clip_grads(z, 0.0)) == 0 and float(z[0].abs().sum()) == 0


def test_one_input_read_twice(scn):
    t = make([5000], [F], 8)[0]
    a, b = torch.empty_like(t), torch.empty_like(t)
    exact = [f64(t)] * 2
    check(scn.clip_grads([t, t], 3.0, out=[a, b]), [a, b], exact, 3.0)
    # in place it would be scaled twice, or read while it is written
    with pytest.raises(scn.ScnError, match="overlap"):
        scn.clip_grads([t, t], 3.0)
    with pytest.raises(scn.ScnError, match="overlap"):
        scn.clip_grads([t[:3000], t[2999:]], 3.0)
    with pytest.raises(scn.ScnError, match="overlap"):
        scn.clip_grads([t[:2000], t[2000:4000]], 3.0, out=[t[:2000], t[1000:3000]])


def test_graph(scn):
    grads = make([3000] * 140 + [70001], [F, B], 9)
    source = [t.clone() for t in grads]
    scn.clip_grads(grads, 1.0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        norm = scn.clip_grads(grads, 1.0)
    for i in range(3):
        for t, s in zip(grads, source):
            t.copy_(s * (i + 0.25))
        want = [t.clone() for t in grads]
        wn = scn.clip_grads(want, 1.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, wn) and all(torch.equal(a, b) for a, b in zip(grads, want))
