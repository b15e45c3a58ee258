"""The attention layer: gradients of all its parameters and its input against
differences of a 64-bit forward, both types; streams against the batch."""
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


def f64(t):
    torch.cuda.synchronize()
    return t.detach().double().cpu().numpy()


def forward64(layer, params, coords, lens, x):
    """The layer's forward in 64 bits, from its formulas."""
    H, K, D = layer.heads, layer.kv, layer.dim
    qkv = (x @ params["Wqkv"][0]).reshape(len(x), H + 2 * K, D)
    freq = f64(layer.freq)
    q, _ = ref.norm_rotate(qkv[:, :H], params["wq"], coords, freq, layer.sections, 1e-6, False)
    k, _ = ref.norm_rotate(qkv[:, H:H + K], params["wk"], coords, freq, layer.sections, 1e-6, False)
    o = ref.attention(q, k, qkv[:, H + K:], lens, layer.left, layer.right, layer.sinks, D ** -0.5,
                      False)["o"][0]
    return x + o.reshape(len(x), H * D) @ params["Wo"][0]


def make(scn, dtype, lens, **kw):
    from paper_1505_02890_amd.attention import SiteAttention, _strokes
    layer = SiteAttention(32, heads=4, kv=2, dim=16, dtype=dtype, **kw)
    g = torch.Generator().manual_seed(3)
    for name in ("wq", "wk"):
        layer.params[name].copy_(1 + 0.3 * torch.randn(16, generator=g))
    coords, sites = _strokes(lens, 40, 5)
    x = torch.randn(len(coords), 32, generator=g).cuda()
    return layer, coords, sites, scn.site_ranges(coords, len(lens)), x


def test_layer_and_gradients(scn):
    # fp32.  Forward: products of up to 64 terms, a softmax and a norm in fp32, some 1e-6 of
    # values of size 1 to 5; the bound leaves a factor of ten.  Gradients: against central
    # differences along random directions; the differences' own error is h^2 = 1e-8 of
    # their third derivatives and 1e-16 / h, the gradient's some 1e-6 of its terms.
    lens = [70, 1, 45]
    layer, coords, sites, ranges, x = make(scn, torch.float32, lens, left=20, right=0, sinks=2)
    y, saved = layer.forward(sites, coords, ranges, x)
    P = {n: f64(w) for n, w in layer.params.items()}
    c = coords.cpu().numpy()
    assert np.abs(f64(y) - forward64(layer, P, c, lens, f64(x))).max() <= 5e-5
    dy = torch.randn(y.shape, generator=torch.Generator().manual_seed(9)).cuda()
    dx, grads = layer.backward(saved, dy)
    G, X = f64(dy), f64(x)
    rng = np.random.default_rng(1)
    h = 1e-4
    for name in ("x",) + tuple(P):
        for _ in range(2):
            e = rng.standard_normal(X.shape if name == "x" else P[name].shape)

            def loss(s):
                p = dict(P)
                if name != "x":
                    p[name] = P[name] + s * e
                return (forward64(layer, p, c, lens, X + s * e if name == "x" else X) * G).sum()

            want = (loss(h) - loss(-h)) / (2 * h)
            got = f64(dx if name == "x" else grads[name]).reshape(e.shape)
            assert abs((got * e).sum() - want) <= 2e-5 * np.abs(got * e).sum(), name


def test_layer_in_bf16(scn):
    # q, k, v, o and the gradients between them are rounded to bf16 (2^-8 each): a few
    # percent of the attention's share of a value, in root mean square under 2%
    lens = [300, 200]
    layer, coords, sites, ranges, x = make(scn, torch.bfloat16, lens, left=64, right=64, sinks=1)
    y, saved = layer.forward(sites, coords, ranges, x)
    P = {n: f64(w) for n, w in layer.params.items()}
    want = forward64(layer, P, coords.cpu().numpy(), lens, f64(x)) - f64(x)
    assert np.linalg.norm(f64(y) - f64(x) - want) <= 0.02 * np.linalg.norm(want)
    exact, ec, es, er, ex = make(scn, torch.float32, lens, left=64, right=64, sinks=1)
    dy = torch.randn(y.shape, generator=torch.Generator().manual_seed(9)).cuda()
    dx, grads = layer.backward(saved, dy)
    rx, rg = exact.backward(exact.forward(es, ec, er, ex)[1], dy)
    for name in grads:
        a, b = f64(grads[name]), f64(rg[name])
        assert np.linalg.norm(a - b) <= 0.05 * np.linalg.norm(b), name
    assert np.linalg.norm(f64(dx - rx)) <= 0.02 * np.linalg.norm(f64(rx - dy))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_streams_follow_the_batch(scn, dtype):
    # two strokes, the first points as a batch, the others one by one
    lens, past = [90, 90], 50
    layer, coords, sites, ranges, x = make(scn, dtype, lens, left=25, right=0, sinks=3)
    y, _ = layer.forward(sites, coords, ranges, x)
    y, x = y.view(2, 90, -1), x.view(2, 90, -1)
    c = coords.view(2, 90, -1)
    from paper_1505_02890_amd.attention import _strokes
    head = c[:, :past].reshape(-1, 4).contiguous()
    _, few = _strokes([past, past], 40, 5)
    _, saved = layer.forward(few, head, scn.site_ranges(head, 2),
                             x[:, :past].reshape(2 * past, -1).contiguous())
    st = layer.open(2, 3 + 26)
    layer.fill(st, saved)
    assert st.length.tolist() == [past, past]
    tol = 2e-5 if dtype == torch.float32 else 0.06  # (bf16: some roundings of 2^-8 of 1 to 5)
    for t in range(past, 90):
        out = layer.step(st, c[:, t].contiguous(), x[:, t].contiguous())
        assert float((out - y[:, t]).abs().max()) <= tol, t
    assert st.length.tolist() == [90, 90]


def test_example_learns(scn, capsys):
    from paper_1505_02890_amd import attention
    attention.main(steps=21)
    out = capsys.readouterr().out
    loss = [float(line.split()[-1]) for line in out.splitlines() if line.startswith("step")]
    assert loss[-1] < 0.8 * loss[0]
    assert float(out.split("within ")[1].split()[0]) <= 1e-4
