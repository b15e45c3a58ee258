"""Attention's gradients in bf16 where rows see few keys: dq and dk are differences
of nearly equal terms there, which the rounding of o to bf16 must not reach."""
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


def inputs(lens, H, K, D, seed):
    g = torch.Generator().manual_seed(seed)
    n = sum(lens)
    t = [torch.randn(n, h, D, generator=g).to(torch.bfloat16).cuda() for h in (H, K, K, H)]
    ranges = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    return t, ranges


def backward(scn, t, ranges, **how):
    q, k, v, do = t
    o, lse = scn.attn_fwd(q, k, v, ranges, **how)
    return scn.attn_bwd(q, k, v, o, lse, do, ranges, **how)


# Two independent roundings to bf16, of dS and of the result, each of at most 2^-8 / sqrt(3)
# (an error spread evenly over half a unit) in the root mean square; the sums are in fp32.
FROBENIUS = 2 ** 0.5 * 2.0 ** -8 / 3 ** 0.5


@pytest.mark.parametrize("D", [16, 32, 64, 96, 128])
@pytest.mark.parametrize("left,right,lens", [
    (1, 0, [700, 333]), (0, 1, [700, 333]), (1, 1, [1031]), (3, 0, [5, 900]),
    (None, 0, [2] * 300), (None, None, [3, 2] * 150)])
def test_few_keys(scn, D, left, right, lens):
    H, K = 4, 2
    t, ranges = inputs(lens, H, K, D, 7)
    got = backward(scn, t, ranges, left=left, right=right)
    q, k, v, do = (x.double().cpu().numpy() for x in t)
    want = ref.attention(q, k, v, lens, left, right, 0, D ** -0.5, True, do)
    for name in ("dq", "dk", "dv"):
        x, w = got[name].double().cpu().numpy(), want[name][0]
        assert np.linalg.norm(x - w) <= FROBENIUS * np.linalg.norm(w), name


# A row that sees one key learns nothing through its score.  What o's rounding leaves of
# <do, o> (half a unit of each product) is taken back but for a rounding of its own.
@pytest.mark.parametrize("D", [16, 64, 72, 128])
@pytest.mark.parametrize("left,right,lens", [(0, 0, [500]), (None, None, [1] * 70)])
def test_one_key(scn, D, left, right, lens):
    t, ranges = inputs(lens, 2, 2, D, 8)
    got = backward(scn, t, ranges, left=left, right=right)
    q, k, v, do = (x.double().cpu().numpy() for x in t)
    most = 2.0 ** -15 * D ** -0.5 * (np.abs(do * v).sum(-1, keepdims=True))
    assert (np.abs(got["dq"].double().cpu().numpy()) <= most * np.abs(k)).all()
    assert (np.abs(got["dk"].double().cpu().numpy()) <= most * np.abs(q)).all()


# Infinite values of a key change nothing for the rows that do not see it, nor for the
# keys that only such rows see.
@pytest.mark.parametrize("D", [64, 96])
def test_masked_infinity_with_few_keys(scn, D):
    n, at = 150, 70
    t, ranges = inputs([n], 2, 1, D, 9)
    q, k, v, do = (x.double().cpu().numpy() for x in t)
    want = ref.attention(q, k, v, [n], 1, 0, 0, D ** -0.5, True, do)
    t[2][at] = torch.inf
    got = backward(scn, t, ranges, left=1, right=0)
    rows = np.abs(np.arange(n) - at) > 1
    for name in ("dq", "dk", "dv"):
        x, (w, b) = got[name].double().cpu().numpy(), want[name]
        assert (np.abs(x - w) <= b)[rows].all(), name
