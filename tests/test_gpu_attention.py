"""Attention among the active sites on the GPU: norm and rotation, attention with
windows and sinks (forward, backward), steps over a ring cache, each against the
64-bit references of ``attention_reference`` with the bounds derived there; masked
infinities and NaN; gradients against differences; refusals."""
from __future__ import annotations

import ctypes

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
    return m


def f64(t):
    torch.cuda.synchronize()
    return t.detach().double().cpu().numpy()


def check(name, got, want, tol):
    got = f64(got)
    assert got.shape == want.shape, name
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.abs(got - want) / tol, 0)), got.shape)
        raise AssertionError(f"{name}: {bad.sum()}/{bad.size} outside their bound, worst at {i}: "
                             f"{got[i]!r} against {want[i]!r}, bound {tol[i]:.3g}")


def bounds(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def qkv(n, H, K, D, dtype, seed, fused=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, H + 2 * K, D, generator=g)
    x[:, :H] *= 1.5
    if fused:  # views of one matrix, as a projection leaves them
        x = x.to(dtype).cuda()
        return x[:, :H], x[:, H:H + K], x[:, H + K:]
    return tuple(t.contiguous().to(dtype).cuda() for t in (x[:, :H], x[:, H:H + K], x[:, H + K:]))


# (lens, Hq, Hk, D, left, right, sinks)
ATTEND = [
    ([1], 1, 1, 8, None, None, 0),
    ([1, 1, 0, 1], 2, 1, 32, 0, 0, 0),
    ([0, 5, 0, 64, 65, 0], 2, 2, 32, None, 0, 0),
    ([127, 128, 129], 4, 1, 64, None, None, 0),
    ([63, 200], 3, 3, 24, 17, 5, 2),
    ([333], 4, 2, 64, 40, 40, 4),
    ([500], 2, 1, 128, 63, 0, 1),
    ([257, 31], 2, 2, 96, 0, 64, 0),
    ([190, 77], 6, 2, 40, 128, 0, 70),       # sinks that overlap the window
    ([700], 1, 1, 16, 3, 2, 300),            # more sinks than have blocks of their own
    ([300], 2, 2, 80, 0, 0, 3),
    ([1100, 2300], 2, 1, 32, 10, 3, 3),      # sinks' queries in several shares
    ([1058], 1, 1, 32, 1023, 0, 35),         # the last share just begins, or does not
    ([1024, 1030], 1, 1, 64, 1000, 4, 40),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attention_and_gradients(scn, case, dtype):
    lens, H, K, D, left, right, sinks = ATTEND[case]
    n = sum(lens)
    q, k, v = qkv(n, H, K, D, TYPES[dtype], 40 + case, fused=case % 2 == 0)
    do = torch.randn(n, H, D, generator=torch.Generator().manual_seed(case)).to(TYPES[dtype]).cuda()
    how = dict(left=left, right=right, sinks=sinks, scale=0.3 if case % 3 == 0 else None)
    o, lse = scn.attn_fwd(q, k, v, bounds(lens), **how)
    d = scn.attn_bwd(q, k, v, o, lse, do, bounds(lens), **how)
    want = ref.attention(f64(q), f64(k), f64(v), lens, left, right, sinks,
                         how["scale"] or D ** -0.5, dtype == "bf16", f64(do))
    for name, got in dict(o=o, lse=lse, **d).items():
        check(name, got, *want[name])
    # the same bits again, on another stream too
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o2, lse2 = scn.attn_fwd(q, k, v, bounds(lens), **how)
        d2 = scn.attn_bwd(q, k, v, o2, lse2, do, bounds(lens), **how)
    s.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert all(torch.equal(d[x], d2[x]) for x in d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_strides_and_outputs(scn, dtype):
    # heads that lie outside rows ([heads, rows, channels]), results into parts of a
    # larger matrix, which keeps the rest
    lens, H, K, D = [150, 60], 4, 2, 32
    n = sum(lens)
    q, k, v = (t.permute(1, 0, 2).contiguous().permute(1, 0, 2)
               for t in qkv(n, H, K, D, TYPES[dtype], 3))
    big = torch.full((n, H + 2 * K + 1, D), 7.0, dtype=TYPES[dtype], device="cuda")
    do = torch.randn(n, H, D, generator=torch.Generator().manual_seed(1)).to(TYPES[dtype]).cuda()
    r = bounds(lens)
    o, lse = scn.attn_fwd(q, k, v, r, left=20, sinks=1, out=big[:, :H])
    want = ref.attention(f64(q), f64(k), f64(v), lens, 20, None, 1, D ** -0.5, dtype == "bf16",
                         f64(do))
    check("o", o, *want["o"])
    assert torch.all(big[:, H:] == 7.0)
    o = o.clone()
    d = scn.attn_bwd(q, k, v, o, lse, do, r, left=20, sinks=1,
                     out=(big[:, :H], big[:, H:H + K], big[:, H + K:H + 2 * K]))
    for x in ("dq", "dk", "dv"):
        check(x, d[x], *want[x])
    assert torch.all(big[:, H + 2 * K:] == 7.0)


def test_rows_outside_the_ranges_are_left(scn):
    q, k, v = qkv(100, 1, 1, 32, torch.float32, 5)
    o = torch.full((100, 1, 32), 7.0, device="cuda")
    r = torch.tensor([20, 50, 80], dtype=torch.int32, device="cuda")
    scn.attn_fwd(q, k, v, r, out=o)
    want = ref.attention(f64(q)[20:80], f64(k)[20:80], f64(v)[20:80], [30, 30], None, None, 0,
                         32 ** -0.5, False)
    check("o", o[20:80], *want["o"])
    assert torch.all(o[:20] == 7.0) and torch.all(o[80:] == 7.0)


@pytest.mark.parametrize("samples", [64, 65, 130, 5000])
def test_many_samples(scn, samples):
    lens = [(7 * i) % 5 for i in range(samples)]
    n = sum(lens)
    q, k, v = qkv(n, 1, 1, 8, torch.float32, 6)
    o, _ = scn.attn_fwd(q, k, v, bounds(lens), right=0)
    want = ref.attention(f64(q), f64(k), f64(v), lens, None, 0, 0, 8 ** -0.5, False)
    check("o", o, *want["o"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_masked_infinities_and_nan_do_not_show(scn, dtype, value):
    # row 100 holds nothing finite; causal with a window of 40 and one sink
    m, H, K, D, left, sinks, at = 300, 2, 1, 64, 40, 1, 100
    t = TYPES[dtype]
    q, k, v = qkv(m, H, K, D, t, 9, fused=False)
    do = torch.randn(m, H, D, generator=torch.Generator().manual_seed(2)).to(t).cuda()
    want = ref.attention(f64(q), f64(k), f64(v), [m], left, 0, sinks, D ** -0.5, dtype == "bf16",
                         f64(do))
    how = dict(left=left, right=0, sinks=sinks)
    r = bounds([m])
    o0, lse0 = scn.attn_fwd(q, k, v, r, **how)
    for x in (q, k, v):
        x[at] = value
    o, lse = scn.attn_fwd(q, k, v, r, **how)
    clean = [i for i in range(m) if not at <= i <= at + left]  # queries that do not see row `at`
    idx = torch.tensor(clean, device="cuda")
    check("o", o[idx], want["o"][0][clean], want["o"][1][clean])
    check("lse", lse[:, idx], want["lse"][0][:, clean], want["lse"][1][:, clean])
    assert not torch.isfinite(o[at]).any()
    # backward of the clean forward with a gradient that is not finite in row `at`: keys
    # outside [at - left, at] but for the sink, and queries but `at`, have clean gradients
    q, k, v = qkv(m, H, K, D, t, 9, fused=False)
    do[at] = value
    d = scn.attn_bwd(q, k, v, o0, lse0, do, r, **how)
    keys = [j for j in range(m) if not at - left <= j <= at and j >= sinks]
    jdx = torch.tensor(keys, device="cuda")
    others = [i for i in range(m) if i != at]
    check("dq", d["dq"][torch.tensor(others, device="cuda")], want["dq"][0][others],
          want["dq"][1][others])
    for x in ("dk", "dv"):
        check(x, d[x][jdx], want[x][0][keys], want[x][1][keys])
    assert torch.isnan(d["dq"][at]).all() and torch.isnan(d["dk"][at - 1]).all()
    assert torch.isnan(d["dk"][0]).all()  # the sink is seen by row `at`
    # a value row that is not finite: queries that do not see it keep their gradients
    do = torch.randn(m, H, D, generator=torch.Generator().manual_seed(2)).to(t).cuda()
    v[at] = value
    d = scn.attn_bwd(q, k, v, o0, lse0, do, r, **how)
    check("dq", d["dq"][idx], want["dq"][0][clean], want["dq"][1][clean])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(scn, dtype):
    # scores of +-10^4: one weight of 1 in each row, and log sums of that size
    q, k, v = qkv(130, 1, 1, 32, TYPES[dtype], 11, fused=False)
    q *= 1000
    want = ref.attention(f64(q), f64(k), f64(v), [130], None, None, 0, 1.0, dtype == "bf16")
    o, lse = scn.attn_fwd(q, k, v, bounds([130]), scale=1.0)
    check("o", o, *want["o"])
    check("lse", lse, *want["lse"])


def test_attention_gradient_against_differences(scn):
    # d loss along a direction, by central differences of the 64-bit forward.  The third
    # derivative term is about h^2 = 1e-8 of the gradient's scale, the differences'
    # rounding 1e-16 / h = 1e-12; the kernel's own bound is in fp32 (1e-5 of the scale).
    lens, H, K, D, left, right, sinks = [90, 41], 2, 1, 24, 12, 6, 2
    n = sum(lens)
    q, k, v = qkv(n, H, K, D, torch.float32, 13, fused=False)
    do = torch.randn(n, H, D, generator=torch.Generator().manual_seed(5)).cuda()
    o, lse = scn.attn_fwd(q, k, v, bounds(lens), left, right, sinks)
    d = scn.attn_bwd(q, k, v, o, lse, do, bounds(lens), left, right, sinks)
    x, G = [f64(t) for t in (q, k, v)], f64(do)
    rng = np.random.default_rng(0)

    def loss(parts):
        return (ref.attention(*parts, lens, left, right, sinks, D ** -0.5, False)["o"][0] * G).sum()

    h = 1e-4
    for i, name in enumerate(("dq", "dk", "dv")):
        for _ in range(3):
            e = rng.standard_normal(x[i].shape)
            up, down = list(x), list(x)
            up[i], down[i] = x[i] + h * e, x[i] - h * e
            want = (loss(up) - loss(down)) / (2 * h)
            got = (f64(d[name]) * e).sum()
            assert abs(got - want) <= 1e-5 * np.abs(f64(d[name]) * e).sum(), name


# (streams, capacity, Hq, Hk, D, left, sinks, lengths)
STEPS = [
    (1, 1, 1, 1, 8, None, 0, [0]),
    (3, 1, 2, 1, 32, None, 0, [0, 1, 7]),
    (4, 9, 2, 2, 24, None, 2, [0, 1, 8, 40]),
    (5, 70, 8, 1, 64, 31, 4, [0, 3, 4, 69, 1000]),
    (2, 300, 16, 1, 32, None, 5, [299, 2 ** 31 - 1]),   # two passes of eight heads
    (3, 257, 3, 3, 80, 0, 0, [5, 256, 257]),
    (2, 64, 4, 2, 128, 5, 63, [70, -3]),
    (1, 5000, 6, 2, 40, None, 1, [4999]),               # split over blocks
    (2, 3001, 4, 4, 128, 2500, 17, [9000, 100]),
    (2, 2048, 2, 1, 16, None, 0, [1, 2047]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(STEPS)))
def test_step(scn, case, dtype):
    B, cap, H, K, D, left, sinks, lengths = STEPS[case]
    t = TYPES[dtype]
    g = torch.Generator().manual_seed(70 + case)
    q, k, v = qkv(B, H, K, D, t, 71 + case)
    # rows that no call may read hold NaN
    kc, vc = (torch.randn(B, cap, K, D, generator=g).to(t).cuda() for _ in range(2))
    length = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    kr, vr = f64(kc), f64(vc)
    if max(lengths) < 10 ** 6:
        want, tol = ref.step(f64(q), f64(k), f64(v), kr, vr, lengths, left, sinks, D ** -0.5,
                             dtype == "bf16")
    else:  # every row of the ring is seen: the same as one full ring further
        ring = cap - sinks
        short = [p if p < cap else sinks + (p - sinks) % ring + ring for p in lengths]
        short = [min(p, sinks + (2 ** 31 - 2 - sinks) % ring + ring) if q_ == 2 ** 31 - 1 else p
                 for p, q_ in zip(short, lengths)]
        want, tol = ref.step(f64(q), f64(k), f64(v), kr, vr, short, left, sinks, D ** -0.5,
                             dtype == "bf16")
    ring = cap - sinks
    reach = ring - 1 if left is None else min(left, ring - 1)
    for b, p in enumerate(lengths):
        p = min(max(p, 0), 2 ** 31 - 2)
        seen = set(range(min(sinks, p + 1)))
        seen |= {sinks + (j - sinks) % ring for j in range(max(sinks, p - reach), p + 1)}
        hidden = [s for s in range(cap) if s not in seen]
        kc[b, hidden], vc[b, hidden] = float("nan"), float("nan")
    now = [p if p < sinks else sinks + (p - sinks) % ring
           for p in (min(max(p, 0), 2 ** 31 - 2) for p in lengths)]
    o = scn.attn_step(q, k, v, kc, vc, length, left=left, sinks=sinks)
    check("o", o, want, tol)
    for b in range(B):
        assert torch.equal(kc[b, now[b]], k[b]) and torch.equal(vc[b, now[b]], v[b])


def test_steps_follow_the_window(scn):
    # a stroke point by point over a ring equals causal attention over all of it
    m, H, K, D, left, sinks = 60, 4, 2, 32, 11, 3
    q, k, v = qkv(m, H, K, D, torch.float32, 90)
    want = ref.attention(f64(q), f64(k), f64(v), [m], left, 0, sinks, D ** -0.5, False)["o"]
    kc, vc = (torch.full((1, sinks + left + 1, K, D), float("nan"), device="cuda")
              for _ in range(2))
    length = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = []
    for i in range(m):
        out.append(scn.attn_step(q[i:i + 1], k[i:i + 1], v[i:i + 1], kc, vc, length, left=left,
                                 sinks=sinks))
        length += 1
    check("o", torch.cat(out), *want)


def test_step_caches_with_strides(scn):
    # [streams, heads, capacity, channels] caches, one matrix for both
    B, cap, H, K, D = 3, 40, 4, 2, 32
    q, k, v = qkv(B, H, K, D, torch.bfloat16, 91)
    both = torch.randn(B, K, cap, 2 * D, generator=torch.Generator().manual_seed(4))
    both = both.to(torch.bfloat16).cuda().permute(0, 2, 1, 3)
    kc, vc = both[..., :D], both[..., D:]
    kr, vr = f64(kc), f64(vc)
    length = [39, 10, 77]
    want, tol = ref.step(f64(q), f64(k), f64(v), kr, vr, length, None, 4, D ** -0.5, True)
    o = scn.attn_step(q, k, v, kc, vc, torch.tensor(length, dtype=torch.int32, device="cuda"),
                      sinks=4)
    check("o", o, want, tol)
    assert np.array_equal(f64(kc), kr) and np.array_equal(f64(vc), vr)


# (rows, Hq, Hk, D, sections, extent, weights)
ROTATE = [
    (1, 1, 1, 8, [4], 5, True),
    (0, 2, 1, 32, [8, 8], 5, True),
    (67, 3, 0, 16, [3, 3, 2], 64, True),
    (130, 4, 2, 24, [3, 3, 3, 3], 512, True),
    (33, 5, 5, 40, [], 64, True),
    (301, 2, 2, 64, [10, 0, 12], 2 ** 31 - 1, True),   # an axis without pairs, pairs not rotated
    (77, 1, 1, 128, [64], 100, False),
    (9000, 9, 6, 80, [14, 13, 13], 300, True),         # four heads share their sines
    (20001, 4, 1, 32, [6, 5, 5], 128, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(ROTATE)))
def test_norm_rotate(scn, case, dtype):
    n, H, K, D, sections, extent, weights = ROTATE[case]
    t = TYPES[dtype]
    g = torch.Generator().manual_seed(case)
    q, k, _ = qkv(n, H, max(K, 1), D, t, 100 + case)
    if K == 0:
        k = None
    rng = np.random.default_rng(case)
    xs = rng.integers(-extent if case % 2 else 0, extent, (n, len(sections)))
    coords = torch.tensor(np.concatenate([np.zeros((n, 1)), xs], 1), dtype=torch.int32).cuda()
    wq, wk = ((1 + 0.3 * torch.randn(D, generator=g)).cuda() if weights else None for _ in range(2))
    freq = scn.rotation_freqs(D, sections)
    dqr = torch.randn(n, H, D, generator=g).to(t).cuda()
    dkr = None if k is None else torch.randn(n, K, D, generator=g).to(t).cuda()
    qr, kr = scn.norm_rotate_fwd(q, k, wq, wk, coords, freq, sections)
    d = scn.norm_rotate_bwd(q, k, wq, wk, coords, freq, sections, dqr, dkr)
    for name, x, w, y, dy in (("q", q, wq, qr, dqr), ("k", k, wk, kr, dkr)):
        if x is None:
            assert y is None and "dk" not in d
            continue
        ry, ty, dx, tx, dw, tw = ref.norm_rotate(f64(x), None if w is None else f64(w),
                                                 coords.cpu().numpy(), f64(freq), sections, 1e-6,
                                                 dtype == "bf16", f64(dy))
        check(name, y, ry, ty)
        check("d" + name, d["d" + name], dx, tx)
        check("dw" + name, d["dw" + name], dw, tw)
    # in place: the same bits
    if k is not None and n:
        q2, k2, g2, h2 = q.clone(), k.clone(), dqr.clone(), dkr.clone()
        d2 = scn.norm_rotate_bwd(q2, k2, wq, wk, coords, freq, sections, g2, h2, out=(g2, h2))
        assert all(torch.equal(d[x], d2[x]) for x in d)
        scn.norm_rotate_fwd(q2, k2, wq, wk, coords, freq, sections, out=(q2, k2))
        assert torch.equal(q2, qr) and torch.equal(k2, kr)


def test_norm_rotate_gradient_against_differences(scn):
    # as above
    n, H, D, sections = 20, 2, 16, [4, 3]
    rng = np.random.default_rng(7)
    x, w, dy = rng.standard_normal((n, H, D)), 1 + 0.3 * rng.standard_normal(D), \
        rng.standard_normal((n, H, D))
    x, w, dy = (a.astype(np.float32).astype(np.float64) for a in (x, w, dy))
    coords = rng.integers(0, 50, (n, 3)).astype(np.int32)
    freq = scn.rotation_freqs(D, sections)

    def dev(a):
        return torch.tensor(a, dtype=torch.float32, device="cuda")

    d = scn.norm_rotate_bwd(dev(x), None, dev(w), None, torch.tensor(coords).cuda(), freq, sections,
                            dev(dy), None)

    def loss(a, b):
        return (ref.norm_rotate(a, b, coords, f64(freq), sections, 1e-6, False)[0] * dy).sum()

    h = 1e-5
    for _ in range(3):
        e, s = rng.standard_normal(x.shape), rng.standard_normal(D)
        want = (loss(x + h * e, w) - loss(x - h * e, w)) / (2 * h)
        assert abs((f64(d["dq"]) * e).sum() - want) <= 1e-5 * np.abs(f64(d["dq"]) * e).sum()
        want = (loss(x, w + h * s) - loss(x, w - h * s)) / (2 * h)
        assert abs((f64(d["dwq"]) * s).sum() - want) <= 1e-5 * np.abs(f64(d["dwq"]) * s).sum()


def test_norm_of_a_zero_row(scn):
    q = torch.zeros(3, 1, 32, device="cuda")
    coords = torch.ones(3, 2, dtype=torch.int32, device="cuda")
    freq = scn.rotation_freqs(32, [16])
    qr, _ = scn.norm_rotate_fwd(q, None, None, None, coords, freq, [16])
    d = scn.norm_rotate_bwd(q, None, None, None, coords, freq, [16], torch.ones_like(q), None)
    assert torch.all(qr == 0) and torch.isfinite(d["dq"]).all()


@pytest.mark.parametrize("counts", [[3], [0, 0, 5], [4, 0, 2, 0], [0]])
def test_site_ranges(scn, counts):
    b = np.repeat(np.arange(len(counts)), counts)
    coords = torch.tensor(np.stack([b, b, b, b], 1).reshape(-1, 4), dtype=torch.int32).cuda()
    want = np.concatenate([[0], np.cumsum(counts)])
    assert f64(scn.site_ranges(coords, len(counts))).tolist() == want.tolist()
    # samples past the batch belong to none of its ranges
    if len(counts) > 1:
        assert f64(scn.site_ranges(coords, len(counts) - 1)).tolist() == want[:-1].tolist()


def test_replayed_graph_equals_the_eager_calls(scn):
    lens, H, K, D = [300, 41], 4, 2, 32
    n = sum(lens)
    q, k, v = qkv(n, H, K, D, torch.bfloat16, 21)
    r, do = bounds(lens), torch.randn(n, H, D, device="cuda").to(torch.bfloat16)
    coords = torch.randint(0, 99, (n, 3), device="cuda").to(torch.int32)
    freq = scn.rotation_freqs(D, [8, 8])
    out = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda")

    def calls():
        qr, kr = scn.norm_rotate_fwd(q, k, None, None, coords, freq, [8, 8])
        o, lse = scn.attn_fwd(qr, kr, v, r, left=30, right=0, sinks=2)
        d = scn.attn_bwd(qr, kr, v, o, lse, do, r, left=30, right=0, sinks=2)
        e = scn.norm_rotate_bwd(q, k, None, None, coords, freq, [8, 8], d["dq"], d["dk"])
        out.copy_(e["dq"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(3):
        q.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        calls()
        torch.cuda.synchronize()
        assert torch.equal(got, out)


def test_bindings_refuse(scn):
    q, k, v = qkv(10, 4, 2, 32, torch.float32, 1)
    r = bounds([10])
    with pytest.raises(ValueError, match="evenly"):
        scn.attn_fwd(q[:, :3], k, v, r)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        scn.attn_fwd(q.half(), k.half(), v.half(), r)
    with pytest.raises(TypeError, match="k must be"):
        scn.attn_fwd(q, k.bfloat16(), v, r)
    with pytest.raises(TypeError, match="CUDA"):
        scn.attn_fwd(q.cpu(), k, v, r)
    with pytest.raises(ValueError, match="shape"):
        scn.attn_fwd(q, k[:9], v, r)
    with pytest.raises(ValueError, match="left"):
        scn.attn_fwd(q, k, v, r, left=-1)
    with pytest.raises(ValueError, match="sinks"):
        scn.attn_fwd(q, k, v, r, sinks=-1)
    with pytest.raises(ValueError, match="contiguous channels"):
        scn.attn_fwd(q.transpose(1, 2).contiguous().transpose(1, 2), k, v, r)
    with pytest.raises(scn.ScnError) as e:
        scn.attn_fwd(q, k, v, r, scale=-1.0)
    assert e.value.status == "invalid"
    with pytest.raises(scn.ScnError) as e:
        scn.attn_fwd(q[..., :20], k[..., :20], v[..., :20], r)
    assert e.value.status == "unsupported"
    with pytest.raises(scn.ScnError) as e:  # rows that are not 16-byte aligned
        scn.attn_fwd(torch.zeros(10, 33, device="cuda")[:, None, 1:], k[:, :1], v[:, :1], r)
    assert e.value.status == "invalid"
    o, lse = scn.attn_fwd(q, k, v, r)
    with pytest.raises(scn.ScnError) as e:
        scn.attn_bwd(q, k, v, o, lse, o, r, ws=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == "workspace"
    kc = torch.zeros(10, 4, 2, 32, device="cuda")
    ln = torch.zeros(10, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="sinks"):
        scn.attn_step(q, k, v, kc, kc.clone(), ln, sinks=4)
    with pytest.raises(ValueError, match="pairs"):
        scn.rotation_freqs(32, [10, 10])
    c = torch.zeros(10, 3, dtype=torch.int32, device="cuda")
    f = scn.rotation_freqs(32, [8, 8])
    with pytest.raises(scn.ScnError) as e:
        scn.norm_rotate_fwd(q, k, None, None, c, f, [10, 10])
    assert e.value.status == "invalid"
    with pytest.raises(ValueError, match="coords"):
        scn.norm_rotate_fwd(q, k, None, None, c, f, [8])


def test_abi_refuses_before_any_launch(scn):
    L = scn.lib()
    i64 = ctypes.c_int64
    assert L.scn_site_ranges(None, 5, 4, 1, None, None) == 1
    assert L.scn_attn_fwd(0, -1, 1, None, 32, 1, 1, None, None, None, 1.0, -1, -1, 0, None, None,
                          None) == 1
    assert L.scn_attn_fwd(7, 1, 1, ctypes.c_void_p(256), 32, 1, 1, None, None, None, 1.0, -1, -1, 0,
                          None, None, None) == 1
    assert b"type" in L.scn_last_error()
    assert L.scn_attn_fwd(0, 2 ** 31, 1, ctypes.c_void_p(256), 32, 1, 1, None, None, None, 1.0, -1,
                          -1, 0, None, None, None) == 4
    assert L.scn_attn_step(0, 1, 2 ** 31, 32, 1, 1, None, None, None, None, None,
                           ctypes.c_void_p(256), 1.0, -1, 0, None, None, 0, None) == 4
    assert L.scn_attn_step_workspace_bytes(0, 1, i64(4), 32, 1, 1, i64(-1), i64(4)) == 0
    assert L.scn_attn_bwd_workspace_bytes(i64(0), 1, 32, 1, 1, i64(-1), i64(0)) == 0
