"""Attention among the active sites as a layer, on the C ABI.

A filter mixes sites two or three lattice steps apart.  This layer lets every
active site of a sample draw on the others, whichever lie far away: the sites
are the tokens, their lattice coordinates the positions, and the order of the
rows the sequence: a rulebook's rows are in key order.  A causal layer along a
stroke needs the points in the order of writing, which a rulebook does not keep
(nor a point that is visited twice): its rows are the points, and its
convolutions, which are 1x1, run on a rulebook over any n distinct sites, as
``_strokes`` has them.

    q, k, v = x Wqkv                      (1x1 convolution, heads side by side)
    q, k    = norm and rotation of each head by the site's coordinates
    o       = attention within the sample, a window of rows and the first ones
    y       = x + o Wo                    (1x1 convolution)

``forward`` and ``backward`` take the sites of a batch (a training step),
``fill`` and ``step`` streams of points that arrive one by one (pen strokes):
a stream keeps its first ``sinks`` points and a ring of its last ones.

Inactive sites take no part: the layer's ground state passes unchanged.  The
products, the norm, the rotation and the attention run in the library's
kernels; this module sequences the calls and adds the residual.

``python -m paper_1505_02890_amd.attention`` trains a layer for some steps on
random strokes and then follows them point by point.
"""
from __future__ import annotations

import math
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

from . import _lib as scn


@dataclass
class Streams:
    """Caches of `streams` strokes: keys and values [streams, capacity, heads, D],
    and the points each holds."""
    k: torch.Tensor
    v: torch.Tensor
    length: torch.Tensor
    sites: "scn.Rulebook"
    capacity: int


class SiteAttention:
    """Random-initialised weights.  ``axes`` lattice axes; ``heads`` query heads
    on ``kv`` heads of keys and values, of ``dim`` channels; ``left``,
    ``right``, ``sinks`` as in ``attn_fwd``; ``dtype`` of the attention
    (float32 or bfloat16; features and weights are float32)."""

    def __init__(self, channels: int, heads: int, kv: int, dim: int, axes: int = 3,
                 left: Optional[int] = None, right: Optional[int] = None, sinks: int = 0,
                 base: float = 100.0, dtype=torch.float32, seed: int = 0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.channels, self.heads, self.kv, self.dim = channels, heads, kv, dim
        self.left, self.right, self.sinks, self.dtype = left, right, sinks, dtype
        p = dim // 2
        self.sections = [p // axes + (1 if a < p % axes else 0) for a in range(axes)]
        self.freq = scn.rotation_freqs(dim, self.sections, base, device)
        wide = (heads + 2 * kv) * dim
        self.params = {
            "Wqkv": (torch.randn(1, channels, wide, generator=g) / math.sqrt(channels)).to(device),
            "wq": torch.ones(dim, device=device), "wk": torch.ones(dim, device=device),
            "Wo": (torch.randn(1, heads * dim, channels, generator=g)
                   / math.sqrt(heads * dim)).to(device)}
        self._zero = torch.zeros(max(channels, heads * dim), device=device)

    def _parts(self, x: torch.Tensor):
        h, k = self.heads, self.kv
        x = x.view(x.shape[0], h + 2 * k, self.dim)
        return x[:, :h], x[:, h:h + k], x[:, h + k:]

    def _project(self, sites, x):
        """(q, k, v) before the norm, views of one matrix of the layer's dtype."""
        qkv, _ = scn.conv_fwd(sites, x, self._zero[:self.channels], self.params["Wqkv"])
        return self._parts(qkv.to(self.dtype))

    def _out(self, sites, o, x):
        o = o.float().view(x.shape[0], self.heads * self.dim)
        y, _ = scn.conv_fwd(sites, o, self._zero[:o.shape[1]], self.params["Wo"])
        return y.add_(x), o

    def forward(self, sites: "scn.Rulebook", coords: torch.Tensor, ranges: torch.Tensor,
                x: torch.Tensor):
        """sites: a rulebook of filter 1, stride 1 over n sites in row order;
        coords int32 [n, 1 + axes], the sample ascending (``out_coords``, or the
        points of strokes); ranges from ``site_ranges``; x [n, channels].  Sites of
        no sample (their first coordinate past the ranges) pass unchanged.
        Returns (y [n, channels], what ``backward`` needs)."""
        p = self.params
        q, k, v = self._project(sites, x)
        qr, kr = scn.norm_rotate_fwd(q, k, p["wq"], p["wk"], coords, self.freq, self.sections)
        # (zeros: rows of no sample are not written, and give nothing)
        o, lse = scn.attn_fwd(qr, kr, v, ranges, self.left, self.right, self.sinks,
                              out=torch.zeros(q.shape, dtype=q.dtype, device=q.device))
        y, of = self._out(sites, o, x)
        return y, (sites, coords, ranges, x, q, k, v, qr, kr, o, lse, of)

    def backward(self, saved, dy: torch.Tensor):
        """Returns (dx, gradients of ``params``)."""
        sites, coords, ranges, x, q, k, v, qr, kr, o, lse, of = saved
        p, n = self.params, x.shape[0]
        out = scn.conv_bwd(sites, of, self._zero[:of.shape[1]], p["Wo"], None, None, dy,
                           need=("dx", "dW"))
        do = out["dx"].to(self.dtype).view(n, self.heads, self.dim)
        dqkv = torch.zeros(n, (self.heads + 2 * self.kv) * self.dim, dtype=self.dtype,
                           device=x.device)
        dq, dk, dv = self._parts(dqkv)
        scn.attn_bwd(qr, kr, v, o, lse, do, ranges, self.left, self.right, self.sinks,
                     out=(dq, dk, dv))
        d = scn.norm_rotate_bwd(q, k, p["wq"], p["wk"], coords, self.freq, self.sections, dq, dk,
                                out=(dq, dk))
        inp = scn.conv_bwd(sites, x, self._zero[:self.channels], p["Wqkv"], None, None,
                           dqkv.float(), need=("dx", "dW"))
        return inp["dx"].add_(dy), {"Wqkv": inp["dW"], "wq": d["dwq"], "wk": d["dwk"],
                                    "Wo": out["dW"]}

    # ----------------------------------------------------------------- streams

    def open(self, streams: int, capacity: int) -> Streams:
        """Empty caches; `capacity` points of each stream, sinks included (the
        window's left + 1 + sinks holds all that a causal window sees).  Of
        causal layers (right = 0) only: a newest point sees none after it."""
        if self.right != 0:
            raise ValueError(f"streams need a causal layer (right=0), this one has {self.right}")
        if capacity <= self.sinks:
            raise ValueError(f"capacity must be above the {self.sinks} sinks, got {capacity}")
        dev = self.freq.device
        k = torch.zeros(streams, capacity, self.kv, self.dim, dtype=self.dtype, device=dev)
        one = torch.zeros(streams, 4, dtype=torch.int32, device=dev)  # one row a stream
        one[:, 0] = torch.arange(streams, device=dev)
        return Streams(k, torch.zeros_like(k), torch.zeros(streams, dtype=torch.int32, device=dev),
                       scn.build_rulebook(one, (max(streams, 1), 1, 1, 1), 1, 1), capacity)

    def fill(self, st: Streams, saved) -> None:
        """The points of a forward (one sample a stream) as the streams' pasts."""
        ranges, v, kr = saved[2].long(), saved[6], saved[8]
        n, ring = v.shape[0], st.capacity - self.sinks
        row = torch.arange(n, device=v.device)
        s = torch.searchsorted(ranges, row, right=True) - 1
        p, m = row - ranges[s], (ranges[1:] - ranges[:-1])[s]
        slot = torch.where(p < self.sinks, p, self.sinks + (p - self.sinks) % ring)
        keep = torch.nonzero((p < self.sinks) | (p >= m - ring))[:, 0]
        st.k[s[keep], slot[keep]] = kr[keep]
        st.v[s[keep], slot[keep]] = v[keep]
        st.length.copy_(ranges[1:] - ranges[:-1])

    def step(self, st: Streams, coords: torch.Tensor, x: torch.Tensor) -> torch.Tensor:
        """One new point of each stream: coords int32 [streams, 1 + axes], x
        [streams, channels].  Returns y [streams, channels]."""
        p = self.params
        q, k, v = self._project(st.sites, x)
        qr, kr = scn.norm_rotate_fwd(q, k, p["wq"], p["wk"], coords, self.freq, self.sections)
        o = scn.attn_step(qr, kr, v, st.k, st.v, st.length, self.left, self.sinks)
        st.length += 1
        return self._out(st.sites, o, x)[0]


def _strokes(lens: Sequence[int], extent: int, seed: int):
    """Walks on the lattice: rows (stroke, x, y, z) in the order of writing, and a
    1x1 rulebook over them (whose sites may repeat along a stroke, so each row
    is a site of its own on a line)."""
    g = torch.Generator().manual_seed(seed)
    rows = []
    for b, m in enumerate(lens):
        steps = torch.zeros(m, 3, dtype=torch.long)
        axis = torch.randint(0, 3, (m,), generator=g)
        steps[torch.arange(m), axis] = 2 * torch.randint(0, 2, (m,), generator=g) - 1
        at = (extent // 2 + steps.cumsum(0)) % extent
        rows.append(torch.cat([torch.full((m, 1), b), at], 1))
    coords = torch.cat(rows).to(torch.int32).cuda()
    line = torch.zeros(len(coords), 4, dtype=torch.int32, device="cuda")
    line[:, 1] = torch.arange(len(coords), device="cuda")
    return coords, scn.build_rulebook(line, (1, len(coords), 1, 1), 1, 1)


def main(steps: int = 30) -> None:
    channels, lens = 64, [400, 250, 317, 1]
    layer = SiteAttention(channels, heads=4, kv=2, dim=32, left=63, right=0, sinks=4)
    coords, sites = _strokes(lens, 64, 1)
    ranges = scn.site_ranges(coords, len(lens))
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(len(coords), channels, generator=g, device="cuda")
    # to learn: each point and the mean of its stroke so far
    want = x + torch.cat([t.cumsum(0) / torch.arange(1, len(t) + 1, device="cuda")[:, None]
                      for t in x.split(lens)])
    for i in range(steps):
        y, saved = layer.forward(sites, coords, ranges, x)
        d = y - want
        _, grads = layer.backward(saved, d * (2.0 / len(d)))
        for name, w in layer.params.items():
            w -= 0.1 * grads[name].view_as(w)
        if i % 10 == 0 or i == steps - 1:
            print(f"step {i:3d}  loss {float(d.square().sum(1).mean()):.4f}", flush=True)
    y, _ = layer.forward(sites, coords, ranges, x)
    first = lens[0]
    st = layer.open(1, 4 + 64)
    out = torch.cat([layer.step(st, coords[i:i + 1], x[i:i + 1]) for i in range(first)])
    print(f"stroke 0 point by point: within {float((out - y[:first]).abs().max()):.2e} of the batch")


if __name__ == "__main__":
    main()
