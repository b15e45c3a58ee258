"""Cross attention between guard rows: inputs stand between rows of NaN, results between rows
that must stay as they are, and so do the rows of no sample within them.  Ranges past the
arrays are clamped; falling ones leave rows undone, and touch nothing outside their
samples."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import block_reference as ref  # noqa: E402
from test_gpu_attention import TYPES, check, f64  # noqa: E402

pytestmark = pytest.mark.gpu

GUARD = 3      # rows in front of and behind each array
HELD = 7.0     # what results hold before the call


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


def between(t, fill):
    """(the larger array, its rows that hold t)"""
    w = torch.full((t.shape[0] + 2 * GUARD, *t.shape[1:]), fill, dtype=t.dtype, device="cuda")
    w[GUARD:-GUARD] = t
    return w, w[GUARD:-GUARD]


def inside(bounds, n):
    """Rows of any sample, by the clamped bounds."""
    at = np.clip(bounds, 0, n)
    rows = np.zeros(n, bool)
    for a, b in zip(at, at[1:]):
        rows[a:b] = True
    return rows


# (rows, states, their bounds, whether the clamped bounds ascend)
RANGES = [
    (50, 60, [0, 20, 20, 50], [0, 10, 40, 60], True),
    (50, 60, [3, 20, 20, 41], [5, 5, 40, 57], True),          # rows of no sample on both sides
    (50, 60, [-5, 20, 30, 99], [-1, 0, 30, 1 << 30], True),
    (50, 60, [0, 60, 20, 50], [0, 10, 70, 60], False),
    (50, 60, [-5, 20, 10, 99], [60, 0, 30, -2], False),
    (50, 60, [50, 50, 50, 50], [0, 0, 0, 0], True),
    (14, 8045, [2, 3, 6, 11], [2, 3002, 8002, 8042], True),   # states in parts
    (14, 8045, [-1, 9, 6, 99], [9000, 2, 8002, 40], False),
    (4005, 60, [2, 2100, 2100, 4002], [1, 21, 50, 58], True),  # rows in parts
    (4005, 60, [4001, 2, 4100, 7], [58, 20, 50, 99], False),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,K,D", [(4, 2, 32), (2, 2, 64), (2, 1, 128)])
@pytest.mark.parametrize("which", range(len(RANGES)))
def test_nothing_outside_the_samples(scn, which, H, K, D, dtype):
    n, m, qb, kb, ascending = RANGES[which]
    g = torch.Generator().manual_seed(which)
    r = lambda *s: torch.randn(*s, generator=g).to(TYPES[dtype]).cuda()  # noqa: E731
    (wq, q), (wk, k), (wv, v), (wg, do) = (between(t, float("nan")) for t in (
        r(n, H, D), r(m, K, D), r(m, K, D), r(n, H, D)))
    keep = [t.clone() for t in (wq, wk, wv, wg)]
    outs = {x: between(torch.full_like(t, HELD), HELD) for x, t in (
        ("o", q), ("dq", q), ("dk", k), ("dv", v))}
    qr, kr = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (qb, kb))
    _, lse = scn.cross_attn_fwd(q, k, v, qr, kr, out=outs["o"][1])
    if not ascending:  # rows undone have no log sum either
        lse.masked_fill_(torch.tensor(~inside(qb, n), device="cuda")[None], 0)
        lse.copy_(torch.where(lse.isfinite() & (lse.abs() < 1e4), lse, torch.zeros_like(lse)))
    scn.cross_attn_bwd(q, k, v, outs["o"][1], lse, do, qr, kr,
                       out=tuple(outs[x][1] for x in ("dq", "dk", "dv")))
    for a, b in zip(keep, (wq, wk, wv, wg)):
        assert torch.equal(a.nan_to_num(), b.nan_to_num()) and torch.equal(a.isnan(), b.isnan())
    rows = {"o": inside(qb, n), "dq": inside(qb, n), "dk": inside(kb, m), "dv": inside(kb, m)}
    for x, (w, t) in outs.items():
        assert bool((w[:GUARD] == HELD).all() and (w[-GUARD:] == HELD).all()), x
        assert bool((t[torch.tensor(~rows[x], device="cuda")] == HELD).all()), x
        if ascending or x == "o":  # (falling bounds: gradients of rows that were not done)
            assert bool(torch.isfinite(t).all()), x
    if not ascending:
        return
    a, b = np.clip(qb, 0, n), np.clip(kb, 0, m)
    want = ref.cross(f64(q)[a[0]:a[-1]], f64(k)[b[0]:b[-1]], f64(v)[b[0]:b[-1]], np.diff(a),
                     np.diff(b), D ** -0.5, dtype == "bf16", f64(do)[a[0]:a[-1]])
    for x, (w, t) in outs.items():
        lo, hi = (a[0], a[-1]) if x in ("o", "dq") else (b[0], b[-1])
        check(x, t[int(lo):int(hi)], *want[x])
    some = np.isfinite(want["lse"][0])
    got = f64(lse)[:, a[0]:a[-1]]
    assert np.array_equal(np.isneginf(got), ~some)
    assert (np.abs(got[some] - want["lse"][0][some]) <= want["lse"][1][some]).all()
