"""A block in which a sample's rows read states of another length, on the C ABI.

``attention.py`` lets the sites of a sample see each other.  This block lets them
read something else of the same sample: the finer level's sites from a pooled level,
a whole scene from a few latent rows, the states of a text from the points of the
stroke that writes it.  With h the rows' norm that the block before has left:

    q, z  = h Wqz                          (1x1 convolution, side by side)
    k, v  = m Wkv                          (of the states m, another number of rows)
    f     = cross attention(q, k, v) Wo    (each sample's rows to its states)
    x'    = alpha x + sigmoid(z) n(f) wf   (the block's norm, gate and residual ...
    h'    = n(x') wh                        ... and the next one's norm, in one pass)

``enter`` forms the first block's h; ``forward`` and ``backward`` take a batch (a
training step, whose gradients ``scn.clip_grads`` clips by their norm), ``open`` and
``step`` streams whose rows arrive one by one while their states stay.

The products, the attention, the norms and the clipping run in the library's
kernels; this module sequences the calls.

``python -m paper_1505_02890_amd.cross`` trains a block for some steps on random
strokes and texts and then follows the strokes point by point.
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import torch

from . import _lib as scn
from .attention import _strokes


@dataclass
class States:
    """Keys and values of streams' states, and the ranges of both sides."""
    k: torch.Tensor
    v: torch.Tensor
    ranges: torch.Tensor
    rows: torch.Tensor
    sites: "scn.Rulebook"


def _line(n: int, device="cuda") -> "scn.Rulebook":
    """A 1x1 rulebook over n rows that are no lattice's sites."""
    line = torch.zeros(n, 4, dtype=torch.int32, device=device)
    line[:, 1] = torch.arange(n, device=device)
    return scn.build_rulebook(line, (1, max(n, 1), 1, 1), 1, 1)


class CrossBlock:
    """Random-initialised weights.  ``channels`` of the rows, ``states`` channels of
    the states; ``heads`` query heads on ``kv`` heads of keys and values, of ``dim``
    channels; ``alpha`` scales the residual; ``dtype`` of the attention (float32 or
    bfloat16; rows, states and weights are float32)."""

    def __init__(self, channels: int, states: int, heads: int, kv: int, dim: int,
                 alpha: float = 1.0, dtype=torch.float32, seed: int = 0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.channels, self.states, self.alpha, self.dtype = channels, states, alpha, dtype
        self.heads, self.kv, self.dim = heads, kv, dim
        self.wide = heads * dim

        def weight(a, b):
            return (torch.randn(1, a, b, generator=g) / math.sqrt(a)).to(device)

        self.params = {"Wqz": weight(channels, self.wide + channels),
                       "Wkv": weight(states, 2 * kv * dim), "Wo": weight(self.wide, channels),
                       "wf": torch.ones(channels, device=device),
                       "wh": torch.ones(channels, device=device)}
        self._zero = torch.zeros(max(channels, states, self.wide), device=device)

    def _conv(self, sites, x, name):
        return scn.conv_fwd(sites, x, self._zero[:x.shape[1]], self.params[name])[0]

    def _queries(self, sites, h):
        qz = self._conv(sites, h, "Wqz")
        q = qz[:, :self.wide].to(self.dtype)
        if qz.shape[1] % 4:  # (the attention's rows lie whole 16 bytes apart)
            q = q.contiguous()
        return q.view(h.shape[0], self.heads, self.dim), qz[:, self.wide:]

    def _keys(self, sites, m):
        kv = self._conv(sites, m, "Wkv").to(self.dtype)
        kv = kv.view(m.shape[0], 2 * self.kv, self.dim)
        return kv[:, :self.kv], kv[:, self.kv:]

    def _leave(self, x, f, z):
        return scn.block_norm_fwd(x, f, z, self.params["wf"], self.params["wh"], self.alpha)

    @staticmethod
    def enter(x: torch.Tensor) -> torch.Tensor:
        """h of the first block: the rows' norm."""
        return scn.block_norm_fwd(x, None, None, None, None, need=("h",))[1]

    @staticmethod
    def enter_bwd(x: torch.Tensor, dx: torch.Tensor, dh: torch.Tensor) -> torch.Tensor:
        """The gradient of x of both its uses."""
        return scn.block_norm_bwd(x, None, None, None, None, dx, dh, need=())["dx"]

    def forward(self, sites: "scn.Rulebook", ranges: torch.Tensor, x: torch.Tensor,
                h: torch.Tensor, state_sites: "scn.Rulebook", state_ranges: torch.Tensor,
                m: torch.Tensor):
        """sites, state_sites: rulebooks of filter 1, stride 1 over the n rows and the
        states, in row order; ranges, state_ranges from ``site_ranges``; x, h
        [n, channels]; m [states, channels of states].  Rows of no sample, and of samples
        without states, read nothing.  Returns (x', h', what ``backward`` needs)."""
        q, z = self._queries(sites, h)
        k, v = self._keys(state_sites, m)
        # (zeros: rows of no sample are not written, and give nothing)
        o, lse = scn.cross_attn_fwd(q, k, v, ranges, state_ranges, out=torch.zeros_like(q))
        of = o.float().view(x.shape[0], self.wide)
        f = self._conv(sites, of, "Wo")
        y, hn = self._leave(x, f, z)
        return y, hn, (sites, ranges, x, h, state_sites, state_ranges, m, q, z, k, v, o, lse, of, f)

    def backward(self, saved, dy: torch.Tensor, dh: torch.Tensor):
        """dy, dh: gradients of x' and h' (dh None: h' has no use).  Returns (dx, dh of
        the block's h, dm, gradients of ``params``)."""
        sites, ranges, x, h, state_sites, state_ranges, m, q, z, k, v, o, lse, of, f = saved
        p, n = self.params, x.shape[0]
        d = scn.block_norm_bwd(x, f, z, p["wf"], p["wh"], dy, dh, self.alpha)
        out = self._conv_bwd(sites, of, "Wo", d["df"])
        dqz = torch.zeros(n, self.wide + self.channels, device=x.device)
        dqz[:, self.wide:] = d["dz"]
        dkv = torch.zeros(m.shape[0], 2 * self.kv, self.dim, dtype=self.dtype, device=x.device)
        g = scn.cross_attn_bwd(q, k, v, o, lse, out["dx"].to(self.dtype).view(q.shape), ranges,
                               state_ranges, out=(torch.zeros_like(q), dkv[:, :self.kv],
                                                  dkv[:, self.kv:]))
        dqz[:, :self.wide] = g["dq"].view(n, self.wide)
        rows = self._conv_bwd(sites, h, "Wqz", dqz)
        states = self._conv_bwd(state_sites, m, "Wkv", dkv.float().view(m.shape[0], -1))
        return d["dx"], rows["dx"], states["dx"], {"Wqz": rows["dW"], "Wkv": states["dW"],
                                                   "Wo": out["dW"], "wf": d["dwf"],
                                                   "wh": d["dwh"]}

    def _conv_bwd(self, sites, x, name, dy):
        return scn.conv_bwd(sites, x, self._zero[:x.shape[1]], self.params[name], None, None, dy,
                            need=("dx", "dW"))

    # ----------------------------------------------------------------- streams

    def open(self, state_sites: "scn.Rulebook", state_ranges: torch.Tensor,
             m: torch.Tensor) -> States:
        """The states of streams, one range of them a stream."""
        k, v = self._keys(state_sites, m)
        n = state_ranges.shape[0] - 1
        rows = torch.arange(n + 1, dtype=torch.int32, device=m.device)
        return States(k, v, state_ranges, rows, _line(n, m.device))

    def step(self, st: States, x: torch.Tensor, h: torch.Tensor):
        """One row of each stream: x, h [streams, channels].  Returns (x', h')."""
        q, z = self._queries(st.sites, h)
        o, _ = scn.cross_attn_fwd(q, st.k, st.v, st.rows, st.ranges)
        return self._leave(x, self._conv(st.sites, o.float().view(x.shape[0], self.wide), "Wo"), z)


def main(steps: int = 30) -> None:
    channels, lens, texts = 64, [400, 250, 317, 1], [11, 7, 0, 5]
    block = CrossBlock(channels, channels, heads=4, kv=2, dim=32)
    coords, sites = _strokes(lens, 64, 1)
    ranges = scn.site_ranges(coords, len(lens))
    state_sites = _line(sum(texts))
    state_ranges = torch.tensor([0] + texts, device="cuda").cumsum(0).to(torch.int32)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(len(coords), channels, generator=g, device="cuda")
    m = torch.randn(sum(texts), channels, generator=g, device="cuda")
    # to learn: each point and the mean of its stroke's text (one stroke has none)
    mean = [t.mean(0) if len(t) else torch.zeros(channels, device="cuda") for t in m.split(texts)]
    want = x + torch.stack(mean).repeat_interleave(torch.tensor(lens, device="cuda"), 0)
    h = block.enter(x)
    for i in range(steps):
        y, _, saved = block.forward(sites, ranges, x, h, state_sites, state_ranges, m)
        d = y - want
        _, _, _, grads = block.backward(saved, d * (2.0 / len(d)), None)
        norm = scn.clip_grads(list(grads.values()), 1.0)
        for name, w in block.params.items():
            w -= 0.1 * grads[name].view_as(w)
        if i % 10 == 0 or i == steps - 1:
            print(f"step {i:3d}  loss {float(d.square().sum(1).mean()):.4f}  "
                  f"gradient norm {float(norm):.3f}", flush=True)
    y, _, _ = block.forward(sites, ranges, x, h, state_sites, state_ranges, m)
    # the strokes point by point, while each has one
    st = block.open(state_sites, state_ranges, m)
    first = ranges[:-1].long()
    far = 0.0
    for i in range(max(lens)):
        at = torch.minimum(first + i, ranges[1:].long() - 1)
        got, _ = block.step(st, x[at], h[at])
        far = max(far, float((got - y[at]).abs().max()))
    print(f"strokes point by point: within {far:.2e} of the batch")


if __name__ == "__main__":
    main()
