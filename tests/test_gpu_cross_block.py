"""The block of ``cross.py``: gradients of all its parameters, its rows and its states
against differences of a 64-bit forward; two blocks in a chain with clipped gradients;
rows of no sample and samples without states; streams against the batch; a captured
training step; the example runs."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import block_reference as ref  # noqa: E402
from test_gpu_attention import f64  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


def forward64(block, params, qlens, klens, x, h, m):
    """The block's forward in 64 bits, from its formulas."""
    H, K, D = block.heads, block.kv, block.dim
    qz = h @ params["Wqz"][0]
    kv = (m @ params["Wkv"][0]).reshape(len(m), 2 * K, D)
    o = ref.cross(qz[:, :H * D].reshape(-1, H, D), kv[:, :K], kv[:, K:], qlens, klens, D ** -0.5,
                  False)["o"][0]
    f = o.reshape(len(x), H * D) @ params["Wo"][0]
    out = ref.block(x, f, qz[:, H * D:], params["wf"], params["wh"], block.alpha, 1e-6, False, False)
    return out["y"][0], out["h"][0]


def make(scn, dtype, qlens, klens, seed=3, alpha=0.9):
    from paper_1505_02890_amd.cross import CrossBlock, _line
    block = CrossBlock(24, 16, heads=4, kv=2, dim=16, alpha=alpha, dtype=dtype, seed=seed)
    g = torch.Generator().manual_seed(seed)
    for name in ("wf", "wh"):
        block.params[name].copy_(1 + 0.3 * torch.randn(24, generator=g))
    r = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    b = lambda lens: torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()  # noqa: E731
    x, m = r(sum(qlens), 24), r(sum(klens), 16)
    return block, _line(sum(qlens)), b(qlens), x, _line(sum(klens)), b(klens), m, r


LENS = ([5, 0, 9, 3], [7, 4, 0, 40])


def test_block_and_gradients(scn):
    # fp32: products of up to 64 terms, a softmax and three norms in fp32, some 1e-6 of values
    # of size 1 to 5; the bounds leave a factor of ten.  Differences at 1e-5 add 1e-10 / 1e-5
    # of rounding in 64 bits and as much of curvature.
    block, sites, qr, x, ms, kr, m, r = make(scn, torch.float32, *LENS)
    h = block.enter(x)
    y, hn, saved = block.forward(sites, qr, x, h, ms, kr, m)
    params = {k: f64(w) for k, w in block.params.items()}
    X, Hh, M = f64(x), f64(h), f64(m)
    wy, wh = forward64(block, params, *LENS, X, Hh, M)
    assert np.abs(f64(y) - wy).max() < 2e-5 and np.abs(f64(hn) - wh).max() < 2e-5
    dy, dh = r(*y.shape), r(*y.shape)
    dx, dhin, dm, grads = block.backward(saved, dy, dh)

    def loss(p=params, X=X, Hh=Hh, M=M):
        a, b = forward64(block, p, *LENS, X, Hh, M)
        return (a * f64(dy)).sum() + (b * f64(dh)).sum()

    rng = np.random.default_rng(0)
    for name, got in dict(grads, x=dx, h=dhin, m=dm).items():
        base = {"x": X, "h": Hh, "m": M}.get(name, params.get(name))
        for _ in range(3):
            s = rng.normal(size=base.shape)
            if name in params:
                lo, hi = ({**params, name: base + e * s} for e in (-1e-5, 1e-5))
                num = (loss(p=hi) - loss(p=lo)) / 2e-5
            else:
                key = {"x": "X", "h": "Hh", "m": "M"}[name]
                num = (loss(**{key: base + 1e-5 * s}) - loss(**{key: base - 1e-5 * s})) / 2e-5
            an = float((f64(got).reshape(base.shape) * s).sum())
            size = float(np.abs(f64(got).reshape(base.shape) * s).sum())
            assert abs(an - num) < 1e-5 * (size + 1), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_chain_with_clipped_gradients(scn, dtype):
    # two blocks: the gradient of the loss along the whole clipped step, against 64 bits (fp32)
    from paper_1505_02890_amd.cross import CrossBlock
    block, sites, qr, x, ms, kr, m, r = make(scn, dtype, *LENS)
    second = CrossBlock(24, 16, heads=4, kv=1, dim=16, alpha=1.0, dtype=dtype, seed=9)

    def run():
        h = CrossBlock.enter(x)
        y1, h1, s1 = block.forward(sites, qr, x, h, ms, kr, m)
        y2, _, s2 = second.forward(sites, qr, y1, h1, ms, kr, m)
        d1, dh1, dm2, g2 = second.backward(s2, dy, None)
        d0, dh0, dm1, g1 = block.backward(s1, d1, dh1)
        return y2, CrossBlock.enter_bwd(x, d0, dh0), dm1 + dm2, list(g1.values()) + list(g2.values())

    dy = r(*x.shape)
    y, dx, dm, grads = run()
    before = [f64(g) for g in grads]
    norm = scn.clip_grads(grads, 0.25)
    want = np.sqrt(sum((g * g).sum() for g in before))
    assert abs(float(norm) - want) <= 2.0 ** -23 * want and want > 0.25
    for a, b in zip(grads, before):
        assert np.abs(f64(a) - b * (0.25 / want)).max() <= 2.0 ** -23 * np.abs(b).max()
    if dtype == torch.float32:
        def loss(X, M):
            n = lambda t: t / np.sqrt((t * t).mean(1, keepdims=True) + 1e-6)  # noqa: E731
            p1, p2 = ({k: f64(w) for k, w in b.params.items()} for b in (block, second))
            a, ah = forward64(block, p1, *LENS, X, n(X), M)
            return (forward64(second, p2, *LENS, a, ah, M)[0] * f64(dy)).sum()
        X, M = f64(x), f64(m)
        for got, key in ((dx, 0), (dm, 1)):
            s = np.random.default_rng(key).normal(size=f64(got).shape)
            at = lambda e: loss(X + e * s, M) if key == 0 else loss(X, M + e * s)  # noqa: E731
            num = (at(1e-5) - at(-1e-5)) / 2e-5
            assert abs((f64(got) * s).sum() - num) < 1e-5 * (np.abs(f64(got) * s).sum() + 1)
    # the same bits again
    again = run()
    assert torch.equal(y, again[0]) and torch.equal(dx, again[1])


def test_rows_of_no_sample(scn):
    # rows past the last range keep their residual, gated by nothing
    block, sites, qr, x, ms, kr, m, r = make(scn, torch.float32, *LENS)
    qr = qr.clone()
    qr[-1] = 14  # the last sample ends three rows early
    h = block.enter(x)
    y, _, saved = block.forward(sites, qr, x, h, ms, kr, m)
    assert torch.equal(y[14:], block.alpha * x[14:])
    dx, dh, dm, grads = block.backward(saved, torch.ones_like(x), None)
    assert all(bool(torch.isfinite(t).all()) for t in (dx, dh, dm, *grads.values()))
    assert torch.equal(dx[14:], torch.full_like(dx[14:], block.alpha))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_streams_follow_the_batch(scn, dtype):
    # the same sums by other kernels: fp32 within its rounding (1e-5 of values up to 10), bf16
    # within a rounding of o and of its weights, 2^-7 of values up to 5
    qlens, klens = [6, 4, 9], [700, 0, 33]
    block, sites, qr, x, ms, kr, m, r = make(scn, dtype, qlens, klens)
    h = block.enter(x)
    y, hn, _ = block.forward(sites, qr, x, h, ms, kr, m)
    st = block.open(ms, kr, m)
    first = qr[:-1].long()
    for i in range(4):
        a, b = block.step(st, x[first + i], h[first + i])
        lim = 1e-4 if dtype == torch.float32 else 0.1
        assert float((a - y[first + i]).abs().max()) < lim
        assert float((b - hn[first + i]).abs().max()) < lim


def test_captured_training_step(scn):
    # forward, backward and clipping of the library's calls in a graph, replayed on new inputs,
    # while gradients of an eager pass of the same inputs live
    n, m, H, K, D, C = 300, 900, 4, 2, 32, 96
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    q, k, v, do = r(n, H, D), r(m, K, D), r(m, K, D), r(n, H, D)
    x, f, z, dy, dh, wf, wh = r(n, C), r(n, C), r(n, C), r(n, C), r(n, C), r(C), r(C)
    qr = torch.tensor([0, 1, 170, 300], dtype=torch.int32, device="cuda")
    kr = torch.tensor([0, 800, 800, 900], dtype=torch.int32, device="cuda")
    ins = [q, k, v, do, x, f, z, dy, dh, wf, wh]

    def step():
        o, lse = scn.cross_attn_fwd(q, k, v, qr, kr)
        d = scn.cross_attn_bwd(q, k, v, o, lse, do, qr, kr)
        y, h = scn.block_norm_fwd(x, f, z, wf, wh)
        e = scn.block_norm_bwd(x, f, z, wf, wh, dy, dh)
        grads = [d["dk"], d["dv"], e["dwf"], e["dwh"]]
        norm = scn.clip_grads(grads, 2.0)
        return [o, lse, d["dq"], y, h, e["dx"], e["df"], e["dz"], norm, *grads]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        for t in ins:
            t.copy_(r(*t.shape))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_example(scn, capsys):
    from paper_1505_02890_amd import cross
    cross.main(steps=3)
    said = capsys.readouterr().out
    assert "step   2" in said and "point by point" in said
