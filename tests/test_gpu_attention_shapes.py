"""Attention at the sizes that large calls have: many samples of some hundred rows, so that
every kernel shape that a call may choose takes several tiles, all its waves, windows that
end inside them, sinks and rows that are formed again.  Steps of more query heads than a
pass holds, and norms whose results go past the caches."""
from __future__ import annotations

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
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.abs(got - want) / tol, 0)), got.shape)
        raise AssertionError(f"{name}: {bad.sum()}/{bad.size} outside their bound, worst at {i}: "
                             f"{got[i]!r} against {want[i]!r}, bound {tol[i]:.3g}")


def bounds(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def kernels(call):
    """The attention kernels that a call launches, without their namespaces."""
    from torch.profiler import ProfilerActivity, profile
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA], acc_events=True) as p:
        call()
        torch.cuda.synchronize()
    names = {e.key for e in p.key_averages() if "attn_" in e.key or "norm_" in e.key}
    return {n.replace("void ", "").replace("scn::(anonymous namespace)::", "").split("(")[0]
            .replace(" ", "") for n in names}


# Samples of 40 to 400 rows.  HUNDRED: blocks for four or more a compute unit with four
# key heads, for fewer with one or two; FEW: a handful.
HUNDRED = [40 + (37 * i) % 361 for i in range(130)]
FEW = [330, 1, 0, 259, 128]

# (type, D, Hq, Hk, lens) -> (forward, queries' pass, keys' pass)
SHAPES = {
    ("bf16", 32, 4, 4, 1): ("<1,32,2,1,1>", "<1,32,2,2>", "<1,32,4,1,2>"),
    ("bf16", 64, 4, 4, 1): ("<1,64,4,1,2>", "<1,64,2,2>", "<1,64,4,1,2>"),
    ("bf16", 96, 4, 4, 1): ("<1,96,4,1,1>", "<1,96,4,1>", "<1,96,4,1,2>"),
    ("bf16", 128, 4, 4, 1): ("<1,128,4,1,1>", "<1,128,4,1>", "<1,128,4,1,2>"),
    ("bf16", 24, 4, 2, 1): ("<1,32,2,1,1>", "<1,32,2,2>", "<1,32,2,2,1>"),
    ("bf16", 56, 4, 2, 1): ("<1,64,4,1,2>", "<1,64,2,2>", "<1,64,2,2,1>"),
    ("bf16", 80, 4, 1, 1): ("<1,96,4,1,1>", "<1,96,4,1>", "<1,96,2,2,1>"),
    ("bf16", 120, 4, 1, 1): ("<1,128,4,1,1>", "<1,128,4,1>", "<1,128,2,2,1>"),
    ("bf16", 64, 4, 1, 1): ("<1,64,4,1,2>", "<1,64,2,2>", "<1,64,1,4,1>"),
    ("bf16", 32, 4, 2, 0): ("<1,32,2,2,2>", "<1,32,2,2>", "<1,32,1,4,1>"),
    ("bf16", 64, 4, 2, 0): ("<1,64,2,2,2>", "<1,64,2,2>", "<1,64,1,4,1>"),
    ("bf16", 96, 4, 2, 0): ("<1,96,4,2,1>", "<1,96,2,2>", "<1,96,2,2,1>"),
    ("bf16", 128, 4, 2, 0): ("<1,128,4,2,1>", "<1,128,2,2>", "<1,128,2,2,1>"),
    ("f32", 32, 4, 4, 1): ("<3,32,4,1,1>", "<3,32,2,2>", "<3,32,2,2,1>"),
    ("f32", 64, 4, 4, 1): ("<3,64,4,2,1>", "<3,64,4,2>", "<3,64,2,2,1>"),
    ("f32", 96, 4, 2, 1): ("<3,96,4,1,1>", "<3,96,4,1>", "<3,96,4,1,1>"),
    ("f32", 128, 4, 1, 1): ("<3,128,4,1,1>", "<3,128,4,1>", "<3,128,4,1,1>"),
    ("f32", 32, 4, 2, 0): ("<3,32,4,2,1>", "<3,32,2,2>", "<3,32,2,2,1>"),
}
WINDOWS = [(40, 7, 3), (None, 0, 0), (100, 0, 40), (None, None, 0)]


def inputs(dtype, D, H, K, n, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, H + 2 * K, D, generator=g)
    x[:, :H] *= 1.5
    x = x.to(TYPES[dtype]).cuda()
    do = torch.randn(n, H, D, generator=g).to(TYPES[dtype]).cuda()
    return x[:, :H], x[:, H:H + K], x[:, H + K:], do


@pytest.mark.parametrize("window", range(len(WINDOWS)))
@pytest.mark.parametrize("case", sorted(SHAPES))
def test_shapes(scn, case, window):
    dtype, D, H, K, many = case
    lens = HUNDRED if many else FEW
    left, right, sinks = WINDOWS[window]
    q, k, v, do = inputs(dtype, D, H, K, sum(lens), 17 + window)
    how = dict(left=left, right=right, sinks=sinks)
    r = bounds(lens)
    o, lse = scn.attn_fwd(q, k, v, r, **how)
    d = scn.attn_bwd(q, k, v, o, lse, do, r, **how)
    want = ref.attention(f64(q), f64(k), f64(v), lens, left, right, sinks, D ** -0.5,
                         dtype == "bf16", f64(do))
    for name, got in dict(o=o, lse=lse, **d).items():
        check(name, got, *want[name])


@pytest.mark.parametrize("case", sorted(SHAPES))
def test_shapes_with_infinities(scn, case):
    """Each sample's row 20 holds nothing finite, seen by rows 20 to 30 only."""
    dtype, D, H, K, many = case
    lens = HUNDRED if many else FEW
    left, right, sinks = 10, 0, 2
    q, k, v, do = inputs(dtype, D, H, K, sum(lens), 29)
    want = ref.attention(f64(q), f64(k), f64(v), lens, left, right, sinks, D ** -0.5,
                         dtype == "bf16", f64(do))
    r = bounds(lens)
    first = np.concatenate([[0], np.cumsum(lens)])[:-1]
    place = np.concatenate([np.arange(m) for m in lens])
    at = torch.tensor([b + 20 for b, m in zip(first, lens) if m > 20], device="cuda")
    o, lse = scn.attn_fwd(q, k, v, r, left, right, sinks)
    d = scn.attn_bwd(q, k, v, o, lse, do, r, left, right, sinks)
    for name in ("dq", "dk", "dv"):
        check(name, d[name], *want[name])
    for i, t in enumerate((q, k, v)):
        t[at] = (float("inf"), -float("inf"), float("nan"))[i]
    o2, lse2 = scn.attn_fwd(q, k, v, r, left, right, sinks)
    rows = (place < 20) | (place > 30)
    check("o", o2[torch.tensor(rows, device="cuda")], want["o"][0][rows], want["o"][1][rows])
    check("lse", lse2[:, torch.tensor(rows, device="cuda")], want["lse"][0][:, rows],
          want["lse"][1][:, rows])
    # gradients: rows 20 to 30 have none of their own, sinks see no finite one
    q, k, v, do = inputs(dtype, D, H, K, sum(lens), 29)
    do[at] = float("nan")
    d = scn.attn_bwd(q, k, v, o, lse, do, r, left, right, sinks)
    rows = place != 20
    check("dq", d["dq"][torch.tensor(rows, device="cuda")], want["dq"][0][rows], want["dq"][1][rows])
    rows = ((place < 10) & (place > 1)) | (place > 20)
    for name in ("dk", "dv"):
        check(name, d[name][torch.tensor(rows, device="cuda")], want[name][0][rows],
              want[name][1][rows])
    got = d["dk"][at - 20]  # the first sink
    assert torch.isnan(got).all()


@pytest.mark.parametrize("case", sorted(SHAPES))
def test_calls_choose_the_shapes(scn, case):
    dtype, D, H, K, many = case
    lens = HUNDRED if many else FEW
    q, k, v, do = inputs(dtype, D, H, K, sum(lens), 1)
    r = bounds(lens)
    o, lse = scn.attn_fwd(q, k, v, r, 40, 7, 3)
    ran = kernels(lambda: (scn.attn_fwd(q, k, v, r, 40, 7, 3),
                           scn.attn_bwd(q, k, v, o, lse, do, r, 40, 7, 3)))
    for kernel, shape in zip(("attn_fwd_kernel", "attn_dq_kernel", "attn_dkv_kernel"),
                             SHAPES[case]):
        assert kernel + shape in ran, (kernel, shape, sorted(ran))
    if many:
        parts = 1 if dtype == "bf16" else 3
        assert f"attn_sink_kernel<{parts},{(D + 31) // 32 * 32}>" in ran, sorted(ran)


# (Hq, Hk, D, capacity, length): more query heads on a key head than the 32 columns of a
# product, in one part and in several
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,K,D,cap,length", [(40, 1, 64, 200, 199), (66, 2, 32, 3000, 2999),
                                              (33, 1, 128, 70, 500), (24, 2, 80, 2500, 2400)])
def test_steps_of_many_heads(scn, dtype, H, K, D, cap, length):
    g = torch.Generator().manual_seed(3)
    t = TYPES[dtype]
    q, k, v, kc, vc = (torch.randn(*s, D, generator=g).to(t).cuda()
                       for s in ((1, H), (1, K), (1, K), (1, cap, K), (1, cap, K)))
    want, tol = ref.step(f64(q), f64(k), f64(v), f64(kc), f64(vc), [length], None, 5, D ** -0.5,
                         dtype == "bf16")
    o = scn.attn_step(q, k, v, kc, vc, torch.tensor([length], dtype=torch.int32, device="cuda"),
                      sinks=5)
    check("o", o, want, tol)


@pytest.mark.parametrize("dtype,n,H,K,D", [("bf16", 70001, 4, 4, 64), ("f32", 70003, 6, 2, 32)])
def test_norms_past_the_caches(scn, dtype, n, H, K, D):
    t, sections = TYPES[dtype], [D // 4, D // 4]
    assert n * (H + K) * D * torch.finfo(t).bits // 8 >= 64 << 20  # where the stores change
    g = torch.Generator().manual_seed(4)
    x = torch.randn(n, H + K, D, generator=g).to(t).cuda()
    dy = torch.randn(n, H + K, D, generator=g).to(t).cuda()
    q, k, dqr, dkr = x[:, :H], x[:, H:], dy[:, :H], dy[:, H:]
    w = (1 + 0.3 * torch.randn(D, generator=g)).cuda()
    coords = torch.randint(0, 128, (n, 3), generator=g).to(torch.int32).cuda()
    freq = scn.rotation_freqs(D, sections)
    qr, kr = scn.norm_rotate_fwd(q, k, w, None, coords, freq, sections)
    d = scn.norm_rotate_bwd(q, k, w, None, coords, freq, sections, dqr, dkr)
    c = coords.cpu().numpy()
    for name, a, b, y, z in (("q", q, w, qr, dqr), ("k", k, None, kr, dkr)):
        ry, ty, dx, tx, dw, tw = ref.norm_rotate(f64(a), None if b is None else f64(b), c, f64(freq),
                                                 sections, 1e-6, dtype == "bf16", f64(z))
        check(name, y, ry, ty)
        check("d" + name, d["d" + name], dx, tx)
        check("dw" + name, d["dw" + name], dw, tw)
