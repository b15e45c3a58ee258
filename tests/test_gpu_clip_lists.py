"""Clipping what is no list: generators of gradients and of results, and refusals that name
the tensor."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import f64  # noqa: E402
from test_gpu_clip import B, F, check, make  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def scn():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1505_02890_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("sizes", [[7, 300], [60000, 9, 30001]], ids=["few", "many"])
def test_generators(scn, sizes):
    grads = make(sizes, [F, B], 2)
    exact = [f64(t) for t in grads]
    out = [torch.zeros_like(t) for t in grads]
    check(scn.clip_grads((t for t in grads), 1.5, out=(t for t in out)), out, exact, 1.5)
    layer = torch.nn.ParameterList([torch.nn.Parameter(t.clone()) for t in grads])
    for p, t in zip(layer, grads):
        p.grad = t
    check(scn.clip_grads((p.grad for p in layer.parameters()), 1.5), grads, exact, 1.5)
    assert float(scn.clip_grads(iter([]), 1.0)) == 0


def test_refusals_of_generators(scn):
    a, b = make([40, 50], [F, F], 2)
    with pytest.raises(ValueError, match=r"grads\[1\] must be contiguous"):
        scn.clip_grads((t for t in (a, b[::2])), 1.0)
    with pytest.raises(TypeError, match=r"grads\[0\]"):
        scn.clip_grads((t for t in (None, a)), 1.0)
    with pytest.raises(ValueError, match="out must hold 2 tensors, got 1"):
        scn.clip_grads((t for t in (a, b)), 1.0, out=(t for t in (a,)))
