"""Cross attention at sizes that reach every kernel shape a call may choose, each checked by
name: values, gradients, rows that are formed again (values near the largest, log sums past
8192), infinities that stay in their sample; skewed batches; strides, places and rows of no
sample; bad ranges; offsets past 32 bits; graphs that share a workspace."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import block_reference as ref  # noqa: E402
from test_gpu_attention import TYPES, bounds, check, f64  # noqa: E402
from test_gpu_cross import inputs  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


def kernels(call):
    """The cross attention kernels that a call launches, without their namespaces."""
    from torch.profiler import ProfilerActivity, profile
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA], acc_events=True) as p:
        call()
        torch.cuda.synchronize()
    names = {e.key for e in p.key_averages() if "cross_" in e.key}
    return {n.replace("void ", "").replace("scn::(anonymous namespace)::", "").split("(")[0]
            .replace(" ", "") for n in names}


LENS = {
    "thin": ([1, 3, 0, 5], [3000, 5000, 40, 0]),          # few rows, keys in parts
    "one": ([1] * 7, [90, 1, 33, 0, 64, 200, 31]),        # one row a sample
    "some": ([40, 64, 0, 33, 50], [300, 700, 90, 5, 1200]),
    "rows": ([130, 200, 70], [400, 150, 333]),
    "wide": ([40 + (37 * i) % 361 for i in range(130)], [70 + (53 * i) % 231 for i in range(130)]),
    "text": ([100 + (91 * i) % 401 for i in range(60)], [3 + (17 * i) % 59 for i in range(60)]),
    "text2": ([2100, 1900], [20, 31]),                    # few keys, queries in parts
}

# (type, D, Hq, Hk, lens) -> (forward, queries' pass, keys' pass)
SHAPES = {
    ("bf16", 32, 2, 1, "thin"): ("thin_kernel<32>", "<1,32,1,4,false>", "<1,32,2,2,1,true>"),
    ("bf16", 64, 2, 2, "thin"): ("thin_kernel<64>", "<1,64,1,4,false>", "<1,64,2,2,1,true>"),
    ("bf16", 96, 2, 1, "thin"): ("thin_kernel<96>", "<1,96,1,4,false>", "<1,96,2,2,1,true>"),
    ("bf16", 128, 2, 1, "thin"): ("thin_kernel<128>", "<1,128,1,4,false>", "<1,128,2,2,1,true>"),
    ("bf16", 24, 6, 2, "one"): ("thin_kernel<32>", "<1,32,1,4,false>", "<1,32,2,2,1,true>"),
    ("bf16", 32, 2, 1, "some"): ("fwd_kernel<1,32,2,2,2,false>", "<1,32,2,2,false>",
                                 "<1,32,2,2,1,true>"),
    ("bf16", 56, 4, 2, "rows"): ("fwd_kernel<1,64,2,2,2,false>", "<1,64,2,2,false>",
                                 "<1,64,1,4,1,false>"),
    ("bf16", 80, 4, 2, "rows"): ("fwd_kernel<1,96,4,2,1,false>", "<1,96,2,2,false>",
                                 "<1,96,2,2,1,false>"),
    ("bf16", 128, 4, 2, "rows"): ("fwd_kernel<1,128,4,2,1,false>", "<1,128,2,2,false>",
                                  "<1,128,2,2,1,false>"),
    ("bf16", 32, 4, 4, "wide"): ("fwd_kernel<1,32,4,1,2,false>", "<1,32,2,2,false>",
                                 "<1,32,4,1,2,false>"),
    ("bf16", 64, 4, 4, "wide"): ("fwd_kernel<1,64,4,1,2,false>", "<1,64,2,2,false>",
                                 "<1,64,4,1,2,false>"),
    ("bf16", 96, 4, 4, "wide"): ("fwd_kernel<1,96,4,1,1,false>", "<1,96,4,1,false>",
                                 "<1,96,4,1,2,false>"),
    ("bf16", 128, 4, 4, "wide"): ("fwd_kernel<1,128,4,1,1,false>", "<1,128,4,1,false>",
                                  "<1,128,4,1,2,false>"),
    ("bf16", 64, 4, 2, "wide"): ("fwd_kernel<1,64,4,1,2,false>", "<1,64,2,2,false>",
                                 "<1,64,2,2,1,false>"),
    ("bf16", 32, 4, 2, "text"): ("fwd_kernel<1,32,4,1,2,true>", "<1,32,4,1,true>",
                                 "<1,32,1,4,1,false>"),
    ("bf16", 64, 4, 1, "text"): ("fwd_kernel<1,64,4,1,2,true>", "<1,64,4,1,true>",
                                 "<1,64,1,4,1,false>"),
    ("bf16", 96, 2, 1, "text"): ("fwd_kernel<1,96,4,1,1,true>", "<1,96,4,1,true>",
                                 "<1,96,2,2,1,false>"),
    ("bf16", 128, 2, 2, "text2"): ("fwd_kernel<1,128,4,1,1,true>", "<1,128,4,1,true>",
                                   "<1,128,2,2,1,false>"),
    ("f32", 32, 2, 1, "thin"): ("few_kernel<4,8>", "<3,32,2,2,false>", "<3,32,2,2,1,false>"),
    ("f32", 64, 4, 4, "thin"): ("few_kernel<8,4>", "<3,64,4,2,false>", "<3,64,2,2,1,false>"),
    ("f32", 8, 1, 1, "one"): ("few_kernel<1,1>", "<3,32,4,1,true>", "<3,32,2,2,1,false>"),
    ("f32", 16, 2, 1, "one"): ("few_kernel<2,2>", "<3,32,4,1,true>", "<3,32,2,2,1,false>"),
    ("f32", 128, 4, 1, "one"): ("few_kernel<16,4>", "<3,128,4,1,true>", "<3,128,4,1,1,false>"),
    ("f32", 72, 8, 1, "one"): ("few_kernel<16,8>", "<3,96,4,1,true>", "<3,96,4,1,1,false>"),
    ("f32", 32, 1, 1, "some"): ("fwd_kernel<3,32,2,2,1,false>", "<3,32,2,2,false>",
                                "<3,32,2,2,1,false>"),
    ("f32", 64, 1, 1, "some"): ("fwd_kernel<3,64,2,2,1,false>", "<3,64,4,2,false>",
                                "<3,64,2,2,1,false>"),
    ("f32", 32, 4, 2, "rows"): ("fwd_kernel<3,32,4,2,1,false>", "<3,32,2,2,false>",
                                "<3,32,2,2,1,false>"),
    ("f32", 64, 4, 2, "rows"): ("fwd_kernel<3,64,4,2,1,false>", "<3,64,4,2,false>",
                                "<3,64,2,2,1,false>"),
    ("f32", 96, 4, 2, "rows"): ("fwd_kernel<3,96,4,1,1,false>", "<3,96,4,1,false>",
                                "<3,96,4,1,1,false>"),
    ("f32", 128, 2, 2, "rows"): ("fwd_kernel<3,128,4,1,1,false>", "<3,128,4,1,false>",
                                 "<3,128,4,1,1,false>"),
    ("f32", 32, 4, 4, "wide"): ("fwd_kernel<3,32,4,1,1,false>", "<3,32,2,2,false>",
                                "<3,32,2,2,1,false>"),
    ("f32", 32, 4, 2, "text2"): ("fwd_kernel<3,32,4,1,1,true>", "<3,32,4,1,true>",
                                 "<3,32,1,4,1,false>"),
    ("f32", 64, 4, 2, "text"): ("fwd_kernel<3,64,4,1,1,true>", "<3,64,4,1,true>",
                                "<3,64,2,2,1,false>"),
    ("f32", 96, 2, 1, "text2"): ("fwd_kernel<3,96,4,1,1,true>", "<3,96,4,1,true>",
                                 "<3,96,4,1,1,false>"),
    ("f32", 128, 2, 1, "text2"): ("fwd_kernel<3,128,4,1,1,true>", "<3,128,4,1,true>",
                                  "<3,128,4,1,1,false>"),
}
IDS = ["-".join(map(str, c)) for c in SHAPES]


def compare(scn, q, k, v, do, ql, kl, bf16, skip=()):
    qr, kr = bounds(ql), bounds(kl)
    o, lse = scn.cross_attn_fwd(q, k, v, qr, kr)
    d = scn.cross_attn_bwd(q, k, v, o, lse, do, qr, kr)
    want = ref.cross(f64(q), f64(k), f64(v), ql, kl, q.shape[2] ** -0.5, bf16, f64(do))
    for name, t in dict(o=o, **d).items():
        if name not in skip:
            check(name, t, *want[name])
    some = ~np.isinf(want["lse"][0])
    assert np.array_equal(np.isneginf(f64(lse)), ~some)
    check("lse", lse[torch.tensor(some, device="cuda")], want["lse"][0][some], want["lse"][1][some])
    return o, lse, d


@pytest.mark.parametrize("case", list(SHAPES), ids=IDS)
def test_shapes(scn, case):
    dtype, D, H, K, which = case
    ql, kl = LENS[which]
    q, k, v, do = inputs(sum(ql), sum(kl), H, K, D, TYPES[dtype], 11)
    o, lse, d = compare(scn, q, k, v, do, ql, kl, dtype == "bf16")
    # infinite and NaN states of one sample stay in it
    at = int(np.argmax(kl))
    first, qfirst = sum(kl[:at]), sum(ql[:at])
    k2, v2 = k.clone(), v.clone()
    k2[first + kl[at] // 2] = float("nan")
    v2[first] = float("inf")
    o2, lse2 = scn.cross_attn_fwd(q, k2, v2, bounds(ql), bounds(kl))
    d2 = scn.cross_attn_bwd(q, k2, v2, o2, lse2, do, bounds(ql), bounds(kl))
    qo = torch.ones(sum(ql), dtype=torch.bool, device="cuda")
    qo[qfirst:qfirst + ql[at]] = False
    ko = torch.ones(sum(kl), dtype=torch.bool, device="cuda")
    ko[first:first + kl[at]] = False
    assert torch.equal(o[qo], o2[qo]) and torch.equal(lse[:, qo], lse2[:, qo])
    assert torch.equal(d["dq"][qo], d2["dq"][qo])
    assert torch.equal(d["dk"][ko], d2["dk"][ko]) and torch.equal(d["dv"][ko], d2["dv"][ko])
    assert bool(o2[~qo].isnan().all()) and bool(lse2[:, ~qo].isnan().all())
    assert bool(d2["dq"][~qo].isnan().all())


@pytest.mark.parametrize("case", list(SHAPES), ids=IDS)
def test_rows_formed_again(scn, case):
    dtype, D, H, K, which = case
    ql, kl = LENS[which]
    q, k, v, do = inputs(sum(ql), sum(kl), H, K, D, TYPES[dtype], 12)
    # values near the largest: sums of their terms pass it before the division.  The
    # reference's bounds scale with the values
    big = (v.sign() * (2.0 ** 127 + v.float().abs() * 2.0 ** 123)).to(v.dtype)
    rows = min(3, min(x for x in ql if x))
    o, _ = scn.cross_attn_fwd(q, k, big, bounds(ql), bounds(kl))
    want = ref.cross(f64(q), f64(k), f64(big) * 2.0 ** -20, ql, kl, D ** -0.5, dtype == "bf16")["o"]
    assert bool(torch.isfinite(o).all())
    assert (np.abs(f64(o) * 2.0 ** -20 - want[0]) <= want[1] + 1e-30).all()
    # log sums past 8192: scores of 300 * 30 / sqrt(D) s and more, the same s for all keys of a
    # sample, in some rows of each
    if which in ("wide", "text"):
        return  # (forming all of their rows again takes long)
    s = D ** 0.5
    q, k = q.clone(), k.clone()
    k[:, :, 0] = 32
    at = 0
    for m in ql:
        q[at:at + min(m, rows), :, 0] = float(torch.tensor(300 * s).to(q.dtype))
        at += m
    compare(scn, q, k, v, do, ql, kl, dtype == "bf16")


@pytest.mark.parametrize("case", list(SHAPES), ids=IDS)
def test_calls_choose_the_shapes(scn, case):
    dtype, D, H, K, which = case
    ql, kl = LENS[which]
    q, k, v, do = inputs(sum(ql), sum(kl), H, K, D, TYPES[dtype], 1)
    qr, kr = bounds(ql), bounds(kl)
    o, lse = scn.cross_attn_fwd(q, k, v, qr, kr)
    ran = kernels(lambda: (scn.cross_attn_fwd(q, k, v, qr, kr),
                           scn.cross_attn_bwd(q, k, v, o, lse, do, qr, kr)))
    for prefix, shape in zip(("cross_", "cross_dq_kernel", "cross_dkv_kernel"), SHAPES[case]):
        assert prefix + shape in ran, (prefix + shape, sorted(ran))
    if which == "thin":
        assert any(n.startswith("cross_join_kernel") for n in ran)
        assert any(n.startswith("cross_dq_join_kernel") for n in ran)
    if which == "text2":
        assert any(n.startswith("cross_dkv_join_kernel") for n in ran)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,K,D", [(4, 2, 32), (3, 3, 64), (2, 1, 128)])
def test_skewed_batches(scn, dtype, H, K, D):
    # all of the work in one sample of 150, between empty ones and ones of a row or a state
    for at, many, long in ((0, 3, 7000), (77, 2, 9000), (149, 400, 30), (100, 300, 2000)):
        ql = [1 if i % 7 == 3 else 0 for i in range(150)]
        kl = [1 if i % 5 == 1 else 0 for i in range(150)]
        ql[at], kl[at] = many, long
        q, k, v, do = inputs(sum(ql), sum(kl), H, K, D, TYPES[dtype], at)
        # (rows of one state: dq and dk are 0 by definition, and their bounds those of rounding)
        compare(scn, q, k, v, do, ql, kl, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which", ["thin", "one", "rows", "text2"])
def test_strides_places_and_rows_of_no_sample(scn, dtype, which):
    ql, kl = LENS[which]
    H, K, D = 4, 2, 40
    n, m = sum(ql), sum(kl)
    q, k, v, do = inputs(n, m, H, K, D, TYPES[dtype], 5)
    qr, kr = bounds(ql), bounds(kl)
    o, lse = scn.cross_attn_fwd(q, k, v, qr, kr)
    d = scn.cross_attn_bwd(q, k, v, o, lse, do, qr, kr)

    def apart(t, rows):  # [heads, rows, wider channels], two rows of no sample in front, three behind
        w = torch.full((t.shape[1], rows + 5, D + 24), 7.0, dtype=t.dtype, device="cuda")
        a = w.permute(1, 0, 2)[:, :, 8:8 + D]
        a[2:2 + rows] = t
        return w, a

    (_, q2), (_, do2), (_, k2), (_, v2) = apart(q, n), apart(do, n), apart(k, m), apart(v, m)
    outs = {x: apart(torch.zeros_like(t), r) for x, t, r in (
        ("o", q, n), ("dq", q, n), ("dk", k, m), ("dv", k, m))}
    seven = {x: w.clone() for x, (w, _) in outs.items()}
    qr2, kr2 = qr + 2, kr + 2
    o2, lse2 = scn.cross_attn_fwd(q2, k2, v2, qr2, kr2, out=outs["o"][1])
    d2 = scn.cross_attn_bwd(q2, k2, v2, o2, lse2, do2, qr2, kr2,
                            out=tuple(outs[x][1] for x in ("dq", "dk", "dv")))
    assert torch.equal(o2[2:2 + n], o) and torch.equal(lse2[:, 2:2 + n], lse)
    for x, r in (("dq", n), ("dk", m), ("dv", m)):
        assert torch.equal(d2[x][2:2 + r], d[x])
    for x, (w, a) in outs.items():
        a[2:-3] = 0  # what the calls wrote; all else is as it was
        assert torch.equal(w, seven[x]), x


def test_shared_states(scn):
    # states that all samples share, as the same rows' ranges; and expanded query rows
    q, k, v, do = inputs(12, 200, 4, 2, 32, torch.float32, 2)
    qr = torch.tensor([0, 5, 12], dtype=torch.int32, device="cuda")
    kr = torch.tensor([0, 200, 200], dtype=torch.int32, device="cuda")
    one = q[:1].expand(12, 4, 32)
    o, _ = scn.cross_attn_fwd(one, k, v, qr, kr)
    assert torch.equal(o[:5], o[:1].expand(5, 4, 32)) and float(o[5:].abs().max()) == 0
    with pytest.raises(ValueError, match="expanded"):
        scn.cross_attn_fwd(q, k, v, qr, kr, out=one)


def test_bad_ranges_read_nothing_outside(scn):
    # falling, negative and too large bounds are clamped: some rows are done, none outside
    q, k, v, do = inputs(50, 60, 2, 1, 32, torch.bfloat16, 3)
    for a, b in (([0, 60, 20, 50], [0, 10, 70, 60]), ([-5, 20, 10, 99], [60, 0, 30, -2]),
                 ([50, 50, 50, 50], [0, 0, 0, 0])):
        qr, kr = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (a, b))
        o, lse = scn.cross_attn_fwd(q, k, v, qr, kr, out=torch.zeros_like(q))
        scn.cross_attn_bwd(q, k, v, o, lse, do, qr, kr)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 128])
def test_large_and_equal_scores(scn, dtype, D):
    # whole numbers times powers of two: scores are exact, the largest of a row equal or far
    # from the others, so weights are 1 / (how many are largest) whatever the exponent
    ql, kl, H, K = [2, 40], [600, 70], 2, 1
    rng = np.random.default_rng(4)
    v = torch.tensor(rng.normal(size=(670, K, D)), dtype=torch.float32).to(TYPES[dtype]).cuda()
    for e in (4, 20, 31, 60, 100):
        q = rng.integers(-3, 4, (42, H, D)) * 2.0 ** (e - e // 2)
        k = rng.integers(-3, 4, (670, K, D)) * 2.0 ** (e // 2)
        tq, tk = (torch.tensor(x, dtype=torch.float32).to(TYPES[dtype]).cuda() for x in (q, k))
        o, lse = scn.cross_attn_fwd(tq, tk, v, bounds(ql), bounds(kl), scale=4.0)
        want = ref.cross(q, k, f64(v), ql, kl, 4.0, dtype == "bf16")
        u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        # weights: the exponential, the sum and the division, 64 terms and more of rounding
        assert np.abs(f64(o) - want["o"][0]).max() <= (2 * u + 200 * 2.0 ** -24) * 5, e
        assert np.abs(f64(lse) - want["lse"][0]).max() <= 4 * 2.0 ** -24 * np.abs(
            want["lse"][0]).max() + 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart(scn, dtype):
    # rows 2^22 elements apart, the most that a call takes: the last ones lie 2^32 elements and
    # more from the first
    if torch.cuda.get_device_properties(0).total_memory < 150 << 30:
        pytest.skip("needs some 40 GB of device memory")
    ql, kl, H, K, D, row = [3, 60], [1050, 20], 2, 1, 32, 1 << 22
    n, m = sum(ql), sum(kl)
    g = torch.Generator().manual_seed(1)
    big = torch.empty(m * row, dtype=TYPES[dtype], device="cuda")
    rows = big.view(m, row)[:, :(4 * K + 4 * H) * D].unflatten(1, (4 * K + 4 * H, D))
    rows.copy_(torch.randn(m, 4 * K + 4 * H, D, generator=g))
    k, v, dk, dv, q, do, o, dq = torch.split(rows, [K, K, K, K, H, H, H, H], 1)
    q, do, o, dq = (t[m - n:] for t in (q, do, o, dq))
    assert (m - 1) * row >= 2 ** 32
    want = ref.cross(f64(q), f64(k), f64(v), ql, kl, D ** -0.5, dtype == "bf16", f64(do))
    _, lse = scn.cross_attn_fwd(q, k, v, bounds(ql), bounds(kl), out=o)
    d = scn.cross_attn_bwd(q, k, v, o, lse, do, bounds(ql), bounds(kl), out=(dq, dk, dv))
    for name, t in dict(o=o, lse=lse, **d).items():
        check(name, t, *want[name])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which", ["thin", "rows", "text2"])
def test_graphs_that_share_a_workspace(scn, dtype, which):
    ql, kl = LENS[which]
    H, K, D = 2, 1, 64
    sets = [inputs(sum(ql), sum(kl), H, K, D, TYPES[dtype], s) for s in (1, 2)]
    qr, kr = bounds(ql), bounds(kl)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def call(q, k, v, do):
        o, lse = scn.cross_attn_fwd(q, k, v, qr, kr, ws=ws)
        return [o, lse, *scn.cross_attn_bwd(q, k, v, o, lse, do, qr, kr, ws=ws).values()]

    call(*sets[0])
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(*s))
        graphs.append(g)
    for r in range(3):
        for t in sets[0] + sets[1]:
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(r)).to(t.dtype))
        ws.fill_(255)  # NaN
        want = [call(*s) for s in sets]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
