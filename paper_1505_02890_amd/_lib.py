"""ctypes binding of ``libscn.so`` (the C ABI declared in ``include/scn.h``).

This module only marshals arguments: it checks tensor shapes, dtypes and
devices, allocates the caller-owned outputs and workspaces with PyTorch, and
passes raw device pointers plus the current HIP stream to the library.  Every
step of the computation runs in the library's HIP kernels.  If the library has
not been built the first call raises; there is no fallback.
"""
from __future__ import annotations

import ctypes
import functools
import os
from array import array
from typing import Iterable, Optional, Sequence

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SCN_LIB") or os.path.join(HERE, "libscn.so")

SCN_RELU = 1
# section 1.2, Figure 2: the cubic and square lattices, and the tetrahedral and
# triangular lattices in skewed coordinates (2D lattices: grids with mz = 1)
LATTICES = {"cubic": 0, "tetrahedral": 1, "square": 2, "triangular": 3}
STATUS = {0: "ok", 1: "invalid", 2: "range", 3: "duplicate", 4: "overflow",
          5: "unsupported", 6: "workspace", 7: "hip", 8: "nomem"}

EXPORTED = (
    "scn_rulebook_build", "scn_rulebook_build_lattice", "scn_rulebook_build_nd",
    "scn_rulebook_build_next",
    "scn_rulebook_build_chain",
    "scn_rulebook_get_info", "scn_rulebook_out_coords",
    "scn_rulebook_in_rows", "scn_rulebook_out_rows", "scn_rulebook_offsets",
    "scn_rulebook_export", "scn_rulebook_free", "scn_conv_fwd",
    "scn_conv_bwd_workspace_bytes", "scn_conv_bwd", "scn_maxpool_fwd",
    "scn_maxpool_bwd_workspace_bytes", "scn_maxpool_bwd", "scn_set_allocator",
    "scn_set_dense_forward", "scn_last_error", "scn_version", "scn_conv_fwd_noalloc",
    "scn_conv_fwd_noalloc_max_bytes", "scn_set_kernel_timer", "scn_ceiling_copy",
    "scn_ceiling_mfma_f32", "scn_ceiling_mfma_bf16", "scn_site_ranges", "scn_norm_rotate_fwd",
    "scn_norm_rotate_bwd_workspace_bytes", "scn_norm_rotate_bwd", "scn_attn_fwd",
    "scn_attn_bwd_workspace_bytes", "scn_attn_bwd", "scn_attn_step_workspace_bytes",
    "scn_attn_step", "scn_cross_attn_fwd", "scn_cross_attn_fwd_workspace_bytes",
    "scn_cross_attn_bwd", "scn_cross_attn_bwd_workspace_bytes", "scn_block_norm_fwd",
    "scn_block_norm_bwd_workspace_bytes", "scn_block_norm_bwd", "scn_grad_clip_workspace_bytes",
    "scn_grad_clip",
)

_ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p)
_FREE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p)


class ScnError(RuntimeError):
    def __init__(self, code: int, where: str, message: str):
        super().__init__(f"{where}: status {code} ({STATUS.get(code, '?')}): {message}")
        self.code = code
        self.status = STATUS.get(code, "?")


class _Info(ctypes.Structure):
    _fields_ = [("a_in", ctypes.c_int64), ("a_out", ctypes.c_int64),
                ("n_pairs", ctypes.c_int64), ("K", ctypes.c_int32),
                ("filter", ctypes.c_int32), ("stride", ctypes.c_int32),
                ("input_sorted", ctypes.c_int32), ("in_grid", ctypes.c_int64 * 4),
                ("out_grid", ctypes.c_int64 * 4), ("lattice", ctypes.c_int32),
                ("dense_view", ctypes.c_int32), ("ndim", ctypes.c_int32),
                ("keyed", ctypes.c_int32), ("in_grid_nd", ctypes.c_int64 * 5),
                ("out_grid_nd", ctypes.c_int64 * 5)]


class _Heads(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class _Cache(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("stream", ctypes.c_int64), ("row", ctypes.c_int64),
                ("head", ctypes.c_int64)]


class _Rows(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("row", ctypes.c_int64)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libscn.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"HIP library {LIB_PATH} is missing: build it with "
            "`python -m paper_1505_02890_amd.build` (or __graft_entry__.build())")
    L = ctypes.CDLL(LIB_PATH)
    P, i32, i64, u32, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32,
                            ctypes.c_size_t)
    st, f32 = ctypes.c_int, ctypes.c_float
    sig = {
        "scn_rulebook_build": (st, [P, i64, P, i32, i32, P, ctypes.POINTER(P)]),
        "scn_rulebook_build_lattice": (st, [P, i64, P, i32, i32, i32, P, ctypes.POINTER(P)]),
        "scn_rulebook_build_nd": (st, [P, i64, i32, P, i32, i32, P, ctypes.POINTER(P)]),
        "scn_rulebook_build_next": (st, [P, i32, i32, P, ctypes.POINTER(P)]),
        "scn_rulebook_build_chain": (st, [P, i64, P, i32, i32, P, P, P, ctypes.POINTER(P)]),
        "scn_rulebook_get_info": (st, [P, ctypes.POINTER(_Info)]),
        "scn_rulebook_out_coords": (P, [P]),
        "scn_rulebook_in_rows": (P, [P]),
        "scn_rulebook_out_rows": (P, [P]),
        "scn_rulebook_offsets": (ctypes.POINTER(ctypes.c_int64), [P]),
        "scn_rulebook_export": (st, [P, P, P, P, P]),
        "scn_rulebook_free": (None, [P]),
        "scn_conv_fwd": (st, [P, P, P, P, P, i32, i32, u32, P, P, P]),
        "scn_conv_fwd_noalloc": (st, [P, P, P, P, P, i32, i32, u32, P, P, P]),
        "scn_conv_fwd_noalloc_max_bytes": (sz, []),
        "scn_set_kernel_timer": (st, [P]),
        "scn_ceiling_copy": (st, [P, P, sz, P]),
        "scn_ceiling_mfma_f32": (st, [P, i64, i32, ctypes.POINTER(ctypes.c_double), P]),
        "scn_ceiling_mfma_bf16": (st, [P, i64, i32, ctypes.POINTER(ctypes.c_double), P]),
        "scn_conv_bwd_workspace_bytes": (sz, [P, i32, i32, u32]),
        "scn_conv_bwd": (st, [P, P, P, P, P, P, P, P, i32, i32, u32, P, P, P, P, P, sz, P]),
        "scn_maxpool_fwd": (st, [P, P, P, i32, P, P, P, P]),
        "scn_maxpool_bwd_workspace_bytes": (sz, [P, i32]),
        "scn_maxpool_bwd": (st, [P, P, P, P, i32, P, P, P, sz, P]),
        "scn_site_ranges": (st, [P, i64, i32, i32, P, P]),
        "scn_norm_rotate_fwd": (st, [i32, i64, i32, i32, i32, P, P, P, P, f32, P, i32, P, P, P, P,
                                     P]),
        "scn_norm_rotate_bwd_workspace_bytes": (sz, [i64, i32, i32, i32]),
        "scn_norm_rotate_bwd": (st, [i32, i64, i32, i32, i32, P, P, P, P, f32, P, i32, P, P, P, P,
                                     P, P, P, P, P, sz, P]),
        "scn_attn_fwd": (st, [i32, i64, i32, P, i32, i32, i32, P, P, P, f32, i64, i64, i64, P, P,
                              P]),
        "scn_attn_bwd_workspace_bytes": (sz, [i64, i32, i32, i32, i32, i64, i64]),
        "scn_attn_bwd": (st, [i32, i64, i32, P, i32, i32, i32, P, P, P, P, P, P, f32, i64, i64,
                              i64, P, P, P, P, sz, P]),
        "scn_attn_step_workspace_bytes": (sz, [i32, i32, i64, i32, i32, i32, i64, i64]),
        "scn_attn_step": (st, [i32, i32, i64, i32, i32, i32, P, P, P, P, P, P, f32, i64, i64, P,
                               P, sz, P]),
        "scn_cross_attn_fwd": (st, [i32, i64, i64, i32, P, P, i32, i32, i32, P, P, P, f32, P, P, P,
                                    sz, P]),
        "scn_cross_attn_fwd_workspace_bytes": (sz, [i32, i64, i64, i32, i32, i32, i32]),
        "scn_cross_attn_bwd": (st, [i32, i64, i64, i32, P, P, i32, i32, i32, P, P, P, P, P, P, f32,
                                    P, P, P, P, sz, P]),
        "scn_cross_attn_bwd_workspace_bytes": (sz, [i32, i64, i64, i32, i32, i32, i32]),
        "scn_block_norm_fwd": (st, [i32, i32, i64, i32, P, P, P, P, P, f32, f32, P, P, P]),
        "scn_block_norm_bwd_workspace_bytes": (sz, [i64, i32]),
        "scn_block_norm_bwd": (st, [i32, i32, i64, i32, P, P, P, P, P, f32, f32, P, P, P, P, P, P,
                                    P, P, sz, P]),
        "scn_grad_clip_workspace_bytes": (sz, [i64, i64]),
        "scn_grad_clip": (st, [i64, P, P, ctypes.c_double, P, P, sz, P]),
        "scn_set_allocator": (None, [_ALLOC_FN, _FREE_FN, P]),
        "scn_set_dense_forward": (st, [i64, i32]),
        "scn_last_error": (ctypes.c_char_p, []),
        "scn_version": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def _check(rc: int, where: str):
    if rc != 0:
        msg = lib().scn_last_error().decode(errors="replace")
        raise ScnError(rc, where, msg)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _dev_tensor(t: torch.Tensor, dtype, shape, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


class Rulebook:
    """Owner of a device rulebook built by ``scn_rulebook_build_lattice``
    (or ``scn_rulebook_build_nd`` when ``ndim`` is given).

    ``coords`` is a device int32 [n, 4] tensor of (b, x, y, z) rows; ``grid``
    is (B, mx, my, mz); ``lattice`` is "cubic", "tetrahedral", "square" or
    "triangular".  With ``ndim``, coords is [n, ndim + 1] rows (b, x_1, ..)
    and grid (B, m_1, .., m_ndim) on the hypercubic lattice.  Attributes
    mirror ``scn_rulebook_info``.
    """

    def __init__(self, coords: Optional[torch.Tensor], grid: Sequence[int], filter: int,
                 stride: int, lattice: str = "cubic", prev: Optional["Rulebook"] = None,
                 ndim: Optional[int] = None):
        h = ctypes.c_void_p()
        if ndim is not None:
            n = int(coords.shape[0]) if coords.dim() == 2 else -1
            _dev_tensor(coords, torch.int32, (n, ndim + 1), "coords")
            if lattice != "cubic":
                raise ValueError("sites of ndim coordinates take the hypercubic lattice")
            g = np.ascontiguousarray(np.asarray(grid, dtype=np.int64).reshape(ndim + 1))
            _check(lib().scn_rulebook_build_nd(
                _ptr(coords), n, int(ndim), g.ctypes.data_as(ctypes.c_void_p), int(filter),
                int(stride), ctypes.c_void_p(_stream()), ctypes.byref(h)),
                "scn_rulebook_build_nd")
            device = coords.device
        elif prev is not None:
            # the layer after prev: its sites are prev's active outputs
            _check(lib().scn_rulebook_build_next(prev.handle, int(filter), int(stride),
                                                 ctypes.c_void_p(_stream()), ctypes.byref(h)),
                   "scn_rulebook_build_next")
            device = prev.device
        else:
            n = int(coords.shape[0]) if coords.dim() == 2 else -1
            _dev_tensor(coords, torch.int32, (n, 4), "coords")
            if lattice not in LATTICES:
                raise ValueError(f"lattice must be one of {sorted(LATTICES)}, got {lattice!r}")
            g = np.ascontiguousarray(np.asarray(grid, dtype=np.int64).reshape(4))
            _check(lib().scn_rulebook_build_lattice(
                _ptr(coords), n, g.ctypes.data_as(ctypes.c_void_p), int(filter), int(stride),
                LATTICES[lattice], ctypes.c_void_p(_stream()), ctypes.byref(h)),
                "scn_rulebook_build_lattice")
            device = coords.device
        self._adopt(h, device)

    @classmethod
    def _from_handle(cls, h: ctypes.c_void_p, device) -> "Rulebook":
        rb = cls.__new__(cls)
        rb._adopt(h, device)
        return rb

    def _adopt(self, h: ctypes.c_void_p, device) -> None:
        self._h = h
        self.device = device
        info = _Info()
        _check(lib().scn_rulebook_get_info(self._h, ctypes.byref(info)), "scn_rulebook_get_info")
        self.a_in, self.a_out, self.n_pairs = int(info.a_in), int(info.a_out), int(info.n_pairs)
        self.K, self.filter, self.stride = int(info.K), int(info.filter), int(info.stride)
        self.input_sorted = bool(info.input_sorted)
        self.dense_view = bool(info.dense_view)
        self.lattice = {v: k for k, v in LATTICES.items()}[int(info.lattice)]
        self.ndim, self.keyed = int(info.ndim), bool(info.keyed)
        self.in_grid = tuple(int(v) for v in info.in_grid_nd[:self.ndim + 1])
        self.out_grid = tuple(int(v) for v in info.out_grid_nd[:self.ndim + 1])
        off = lib().scn_rulebook_offsets(self._h)
        self.offsets = np.array([off[k] for k in range(self.K + 1)], dtype=np.int64)

    @property
    def handle(self):
        return self._h

    def close(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _lib is not None:
            _lib.scn_rulebook_free(h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def export(self):
        """(out_coords int32[a_out, ndim+1], in_rows int32[P], out_rows int32[P]) on the
        device."""
        oc = torch.empty((self.a_out, self.ndim + 1), dtype=torch.int32, device=self.device)
        ir = torch.empty(self.n_pairs, dtype=torch.int32, device=self.device)
        orr = torch.empty(self.n_pairs, dtype=torch.int32, device=self.device)
        _check(lib().scn_rulebook_export(self._h, _ptr(oc), _ptr(ir), _ptr(orr),
                                         ctypes.c_void_p(_stream())), "scn_rulebook_export")
        return oc, ir, orr

    def out_coords(self) -> torch.Tensor:
        oc = torch.empty((self.a_out, self.ndim + 1), dtype=torch.int32, device=self.device)
        _check(lib().scn_rulebook_export(self._h, _ptr(oc), None, None,
                                         ctypes.c_void_p(_stream())), "scn_rulebook_export")
        return oc


def build_rulebook(coords: torch.Tensor, grid: Sequence[int], filter: int, stride: int,
                   lattice: str = "cubic") -> Rulebook:
    return Rulebook(coords, grid, filter, stride, lattice)


def build_rulebook_nd(coords: torch.Tensor, grid: Sequence[int], filter: int,
                      stride: int) -> Rulebook:
    """Hypercubic rulebook over sites of ndim = len(grid) - 1 coordinates
    (keyed builder: sorted keys and hash tables)."""
    return Rulebook(coords, grid, filter, stride, ndim=len(grid) - 1)


def next_rulebook(prev: Rulebook, filter: int, stride: int) -> Rulebook:
    """The rulebook of the layer after `prev` (its sites are prev's active
    outputs, on prev's output grid and lattice)."""
    return Rulebook(None, prev.out_grid, filter, stride, prev.lattice, prev=prev)


def conv_fwd(rb: Rulebook, x: torch.Tensor, g_in: torch.Tensor, W: torch.Tensor,
             bias: Optional[torch.Tensor] = None, relu: bool = False,
             y: Optional[torch.Tensor] = None, g_out: Optional[torch.Tensor] = None,
             noalloc: bool = False):
    """Returns (y [a_out, Cout], g_out [Cout]); y and g_out are allocated here
    unless given.  noalloc=True calls scn_conv_fwd_noalloc (the library then
    allocates nothing)."""
    K, Cin, Cout = (int(v) for v in W.shape)
    if K != rb.K:
        raise ValueError(f"W has {K} offsets, rulebook has {rb.K}")
    _dev_tensor(W, torch.float32, (K, Cin, Cout), "W")
    _dev_tensor(x, torch.float32, (rb.a_in, Cin), "x")
    _dev_tensor(g_in, torch.float32, (Cin,), "g_in")
    if bias is not None:
        _dev_tensor(bias, torch.float32, (Cout,), "bias")
    if y is None:
        y = torch.empty((rb.a_out, Cout), dtype=torch.float32, device=x.device)
    _dev_tensor(y, torch.float32, (rb.a_out, Cout), "y")
    if g_out is None:
        g_out = torch.empty(Cout, dtype=torch.float32, device=x.device)
    _dev_tensor(g_out, torch.float32, (Cout,), "g_out")
    name = "scn_conv_fwd_noalloc" if noalloc else "scn_conv_fwd"
    _check(getattr(lib(), name)(rb.handle, _ptr(x), _ptr(g_in), _ptr(W), _ptr(bias), Cin, Cout,
                                SCN_RELU if relu else 0, _ptr(y), _ptr(g_out),
                                ctypes.c_void_p(_stream())), name)
    return y, g_out


def conv_bwd_workspace(rb: Rulebook, Cin: int, Cout: int, relu: bool) -> torch.Tensor:
    n = lib().scn_conv_bwd_workspace_bytes(rb.handle, Cin, Cout, SCN_RELU if relu else 0)
    return torch.empty(max(int(n), 1), dtype=torch.uint8, device=rb.device)


def conv_bwd(rb: Rulebook, x: torch.Tensor, g_in: torch.Tensor, W: torch.Tensor,
             y: Optional[torch.Tensor], g_out: Optional[torch.Tensor], dy: torch.Tensor,
             dg_out: Optional[torch.Tensor] = None, relu: bool = False,
             need=("dx", "dg_in", "dW", "dbias"), ws: Optional[torch.Tensor] = None):
    """Returns a dict with the requested gradients among dx, dg_in, dW, dbias."""
    K, Cin, Cout = (int(v) for v in W.shape)
    _dev_tensor(W, torch.float32, (rb.K, Cin, Cout), "W")
    _dev_tensor(x, torch.float32, (rb.a_in, Cin), "x")
    _dev_tensor(g_in, torch.float32, (Cin,), "g_in")
    _dev_tensor(dy, torch.float32, (rb.a_out, Cout), "dy")
    if relu:
        _dev_tensor(y, torch.float32, (rb.a_out, Cout), "y")
        _dev_tensor(g_out, torch.float32, (Cout,), "g_out")
    if dg_out is not None:
        _dev_tensor(dg_out, torch.float32, (Cout,), "dg_out")
    dev = x.device
    out = {}
    if "dx" in need:
        out["dx"] = torch.empty((rb.a_in, Cin), dtype=torch.float32, device=dev)
    if "dg_in" in need:
        out["dg_in"] = torch.empty(Cin, dtype=torch.float32, device=dev)
    if "dW" in need:
        out["dW"] = torch.empty((K, Cin, Cout), dtype=torch.float32, device=dev)
    if "dbias" in need:
        out["dbias"] = torch.empty(Cout, dtype=torch.float32, device=dev)
    if ws is None:
        ws = conv_bwd_workspace(rb, Cin, Cout, relu)
    _check(lib().scn_conv_bwd(rb.handle, _ptr(x), _ptr(g_in), _ptr(W), _ptr(y), _ptr(g_out),
                              _ptr(dy), _ptr(dg_out), Cin, Cout, SCN_RELU if relu else 0,
                              _ptr(out.get("dx")), _ptr(out.get("dg_in")), _ptr(out.get("dW")),
                              _ptr(out.get("dbias")), _ptr(ws), ws.numel(),
                              ctypes.c_void_p(_stream())), "scn_conv_bwd")
    return out


def maxpool_fwd(rb: Rulebook, x: torch.Tensor, g_in: torch.Tensor):
    """Returns (y [a_out, C], g_out [C], argmax uint8 [a_out, C])."""
    C = int(x.shape[1]) if x.dim() == 2 else -1
    _dev_tensor(x, torch.float32, (rb.a_in, C), "x")
    _dev_tensor(g_in, torch.float32, (C,), "g_in")
    y = torch.empty((rb.a_out, C), dtype=torch.float32, device=x.device)
    g_out = torch.empty(C, dtype=torch.float32, device=x.device)
    am = torch.empty((rb.a_out, C), dtype=torch.uint8, device=x.device)
    _check(lib().scn_maxpool_fwd(rb.handle, _ptr(x), _ptr(g_in), C, _ptr(y), _ptr(g_out), _ptr(am),
                                 ctypes.c_void_p(_stream())), "scn_maxpool_fwd")
    return y, g_out, am


def maxpool_bwd(rb: Rulebook, argmax: torch.Tensor, dy: torch.Tensor,
                dg_out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """Returns (dx [a_in, C], dg_in [C])."""
    C = int(dy.shape[1]) if dy.dim() == 2 else -1
    _dev_tensor(dy, torch.float32, (rb.a_out, C), "dy")
    _dev_tensor(argmax, torch.uint8, (rb.a_out, C), "argmax")
    if dg_out is not None:
        _dev_tensor(dg_out, torch.float32, (C,), "dg_out")
    dx = torch.empty((rb.a_in, C), dtype=torch.float32, device=dy.device)
    dg_in = torch.empty(C, dtype=torch.float32, device=dy.device)
    if ws is None:
        n = lib().scn_maxpool_bwd_workspace_bytes(rb.handle, C)
        ws = torch.empty(max(int(n), 1), dtype=torch.uint8, device=dy.device)
    _check(lib().scn_maxpool_bwd(rb.handle, _ptr(argmax), _ptr(dy), _ptr(dg_out), C, _ptr(dx),
                                 _ptr(dg_in), _ptr(ws), ws.numel(), ctypes.c_void_p(_stream())),
           "scn_maxpool_bwd")
    return dx, dg_in


# ---------------------------------------------------------------------------
# attention among the active sites
# ---------------------------------------------------------------------------

SCN_TYPE = {torch.float32: 0, torch.bfloat16: 1}


def _refuse_rows(t, dtype, device: int, shape, name: str):
    """Why `_rows` or `_cache` did not take a tensor."""
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype not in SCN_TYPE:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    if t.dtype != dtype or t.get_device() != device:
        raise TypeError(f"{name} must be {dtype} on cuda:{device}, got {t.dtype} on {t.device}")
    raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _first(t: torch.Tensor, name: str):
    """The shape [rows, heads, D], type and device that a call's other tensors
    follow."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in SCN_TYPE:
        _refuse_rows(t, None, -1, (), name)
    if t.dim() != 3:
        raise ValueError(f"{name} must have three dimensions, got {tuple(t.shape)}")
    device = t.get_device()
    if device != torch.cuda.current_device():
        raise ValueError(f"{name} is on cuda:{device}, which is not the current device")
    return t.shape, t.dtype, device


def _rows(t: torch.Tensor, dtype, device: int, shape, name: str):
    """ctypes view of a [rows, heads, D] tensor (any strides with contiguous
    channels).  A stride that no element is reached by (one row, one head) is
    passed as 0, whatever torch holds there."""
    if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.is_cuda and
            t.get_device() == device and t.shape == shape):
        _refuse_rows(t, dtype, device, shape, name)
    row, head, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError(f"{name} must have contiguous channels")
    return _Heads(t.data_ptr(), row if shape[0] > 1 else 0, head if shape[1] > 1 else 0)


def _cache(t: torch.Tensor, dtype, device: int, shape, name: str):
    """The same of a [streams, capacity, heads, D] cache."""
    if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.is_cuda and
            t.get_device() == device and t.shape == shape):
        _refuse_rows(t, dtype, device, shape, name)
    stream, row, head, one = t.stride()
    if one != 1 and shape[3] > 1:
        raise ValueError(f"{name} must have contiguous channels")
    return _Cache(t.data_ptr(), stream if shape[0] > 1 else 0, row if shape[1] > 1 else 0,
                  head if shape[2] > 1 else 0)


def _out_rows(t: Optional[torch.Tensor], like: torch.Tensor, shape, name: str):
    """(result, its view), allocated here unless given.  A given result must
    not hold one element twice."""
    if t is None:
        t = torch.empty(shape, dtype=like.dtype, device=like.device)
        return t, _Heads(t.data_ptr(), shape[1] * shape[2], shape[2])
    v = _rows(t, like.dtype, like.get_device(), shape, name)
    if t.numel() and (v.row == 0 and shape[0] > 1 or v.head == 0 and shape[1] > 1):
        raise ValueError(f"{name} must not be expanded")
    return t, v


def _vector(t, dtype, device: int, shape, name: str):
    """Device pointer of a contiguous tensor, or None."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.is_cuda and
            t.get_device() == device and t.shape == shape and t.is_contiguous()):
        _dev_tensor(t, dtype, shape, name)
        raise TypeError(f"{name} must be on cuda:{device}, got {t.device}")
    return t.data_ptr()


def _raw_stream(device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def _bytes(n: int, device) -> torch.Tensor:
    return torch.empty(n or 1, dtype=torch.uint8, device=device)


def site_ranges(coords: torch.Tensor, batch: int) -> torch.Tensor:
    """Row ranges of the samples of key-ordered sites (``scn_site_ranges``):
    int32 [batch + 1] with sample b's rows at [ranges[b], ranges[b + 1]).
    ``coords`` is int32 [n, ndim + 1], the sample first (``Rulebook.out_coords``)."""
    if not isinstance(coords, torch.Tensor) or coords.dim() != 2:
        raise ValueError("coords must be a 2D tensor")
    _dev_tensor(coords, torch.int32, tuple(coords.shape), "coords")
    if batch < 1:
        raise ValueError("batch must be at least 1")
    r = torch.empty(batch + 1, dtype=torch.int32, device=coords.device)
    _check(lib().scn_site_ranges(_ptr(coords), coords.shape[0], coords.shape[1], int(batch),
                                 _ptr(r), ctypes.c_void_p(_stream())), "scn_site_ranges")
    return r


def rotation_freqs(dim: int, sections: Sequence[int], base: float = 100.0,
                   device="cuda") -> torch.Tensor:
    """Frequencies of the rotation for ``norm_rotate_fwd``: float32 [dim / 2],
    the pairs of each axis from 1 radian per lattice step down in a geometric
    series towards 1 / base; pairs past the sections 0."""
    if any(m < 0 for m in sections) or sum(sections) > dim // 2:
        raise ValueError(f"sections {tuple(sections)} must hold at most {dim // 2} pairs")
    f = [float(base) ** (-j / m) for m in sections for j in range(m)]
    return torch.tensor(f + [0.0] * (dim // 2 - len(f)), dtype=torch.float32, device=device)


def _norm_args(q, k, wq, wk, coords, freq, sections):
    shape, dtype, dev = _first(q, "q")
    n, hq, d = shape
    hk = 0
    vk = None
    if k is not None:
        hk = k.shape[1] if k.dim() == 3 else 0
        vk = _rows(k, dtype, dev, (n, hk, d), "k")
    vq = _rows(q, dtype, dev, shape, "q")
    na = len(sections)
    return (SCN_TYPE[dtype], n, d, hq, hk, vq, vk, _vector(wq, torch.float32, dev, (d,), "wq"),
            _vector(wk, torch.float32, dev, (d,), "wk"),
            _vector(coords, torch.int32, dev, (n, na + 1), "coords"), na + 1,
            _vector(freq, torch.float32, dev, (d // 2,), "freq"),
            (ctypes.c_int32 * max(1, na))(*sections), dtype, dev)


def norm_rotate_fwd(q: torch.Tensor, k: Optional[torch.Tensor], wq: Optional[torch.Tensor],
                    wk: Optional[torch.Tensor], coords: torch.Tensor, freq: torch.Tensor,
                    sections: Sequence[int], eps: float = 1e-6, out=(None, None)):
    """Norm of each head's queries and keys and their rotation by the sites'
    coordinates (``scn_norm_rotate_fwd``).  q [n, Hq, D], k [n, Hk, D] (or
    None), float32 or bfloat16, any row and head strides; wq, wk float32 [D] or
    None; coords int32 [n, 1 + axes]; freq float32 [D / 2]; sections the pairs
    of each axis.  Returns (qr, kr), in ``out`` where given (q and k themselves
    may be)."""
    typ, n, d, hq, hk, vq, vk, pwq, pwk, pc, width, pf, sec, _, dev = _norm_args(
        q, k, wq, wk, coords, freq, sections)
    qr, oq = _out_rows(out[0], q, (n, hq, d), "out[0]")
    kr, ok = (None, None) if k is None else _out_rows(out[1], q, (n, hk, d), "out[1]")
    _check(lib().scn_norm_rotate_fwd(typ, n, d, hq, hk, _ref(vq), _ref(vk), pwq, pwk, eps, pc,
                                     width, pf, sec, _ref(oq), _ref(ok), _raw_stream(dev)),
           "scn_norm_rotate_fwd")
    return qr, kr


def norm_rotate_bwd(q: torch.Tensor, k: Optional[torch.Tensor], wq: Optional[torch.Tensor],
                    wk: Optional[torch.Tensor], coords: torch.Tensor, freq: torch.Tensor,
                    sections: Sequence[int], dqr: torch.Tensor, dkr: Optional[torch.Tensor],
                    eps: float = 1e-6, need=("dwq", "dwk"), out=(None, None),
                    ws: Optional[torch.Tensor] = None):
    """Gradients of ``norm_rotate_fwd``: a dict with dq, dk (in ``out`` where
    given; dqr and dkr themselves may be) and the requested ones of dwq, dwk."""
    typ, n, d, hq, hk, vq, vk, pwq, pwk, pc, width, pf, sec, dtype, dev = _norm_args(
        q, k, wq, wk, coords, freq, sections)
    gq = _rows(dqr, dtype, dev, (n, hq, d), "dqr")
    res, gk, ok = {}, None, None
    res["dq"], oq = _out_rows(out[0], q, (n, hq, d), "out[0]")
    if k is not None:
        gk = _rows(dkr, dtype, dev, (n, hk, d), "dkr")
        res["dk"], ok = _out_rows(out[1], q, (n, hk, d), "out[1]")
    pw = {}
    for name in ("dwq", "dwk"):
        if name in need and (name == "dwq" or k is not None):
            res[name] = torch.empty(d, dtype=torch.float32, device=q.device)
            pw[name] = res[name].data_ptr()
    if ws is None:
        ws = _bytes(lib().scn_norm_rotate_bwd_workspace_bytes(n, d, hq, hk) if pw else 0, q.device)
    _check(lib().scn_norm_rotate_bwd(
        typ, n, d, hq, hk, _ref(vq), _ref(vk), pwq, pwk, eps, pc, width, pf, sec, _ref(gq),
        _ref(gk), _ref(oq), _ref(ok), pw.get("dwq"), pw.get("dwk"), ws.data_ptr(), ws.numel(),
        _raw_stream(dev)), "scn_norm_rotate_bwd")
    return res


def _ref(v):
    return None if v is None else ctypes.byref(v)


def _bound(w: Optional[int], name: str) -> int:
    if w is None:
        return -1
    if w < 0:
        raise ValueError(f"{name} must be None (no bound) or at least 0, got {w}")
    return w


def _qkv(q, k, v):
    shape, dtype, dev = _first(q, "q")
    n, hq, d = shape
    hk = k.shape[1] if isinstance(k, torch.Tensor) and k.dim() == 3 else 0
    vq = _rows(q, dtype, dev, shape, "q")
    vk = _rows(k, dtype, dev, (n, hk, d), "k")
    vv = _rows(v, dtype, dev, (n, hk, d), "v")
    if hk < 1 or hq % hk:
        raise ValueError(f"{hq} query heads cannot share {hk} key heads evenly")
    return dtype, dev, n, hq, hk, d, vq, vk, vv


def _attn_args(ranges, dev, left, right, sinks, scale, d):
    batch = ranges.shape[0] - 1 if isinstance(ranges, torch.Tensor) and ranges.dim() == 1 else 0
    if batch < 1:
        raise ValueError("ranges must hold at least two bounds")
    pr = _vector(ranges, torch.int32, dev, (batch + 1,), "ranges")
    if sinks < 0:
        raise ValueError(f"sinks must be at least 0, got {sinks}")
    return (batch, pr, d ** -0.5 if scale is None else scale, _bound(left, "left"),
            _bound(right, "right"))


def attn_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, ranges: torch.Tensor,
             left: Optional[int] = None, right: Optional[int] = None, sinks: int = 0,
             scale: Optional[float] = None, out: Optional[torch.Tensor] = None):
    """Attention within each sample (``scn_attn_fwd``).  q [n, Hq, D], k and v
    [n, Hk, D], float32 or bfloat16, any row and head strides; ``ranges`` from
    ``site_ranges``.  Row i of a sample sees row j if j <= i + right and
    (j >= i - left or j < sinks); None is no bound, right=0 causal.  scale is
    D ** -0.5 unless given.  Returns (o [n, Hq, D], lse float32 [Hq, n]).  Rows
    outside every range (of samples past the batch) are not written: they hold
    what ``out`` held, or nothing that means anything.  ``out`` may not overlap q, k or v."""
    dtype, dev, n, hq, hk, d, vq, vk, vv = _qkv(q, k, v)
    batch, pr, scale, l, r = _attn_args(ranges, dev, left, right, sinks, scale, d)
    o, vo = _out_rows(out, q, (n, hq, d), "out")
    lse = torch.empty((hq, n), dtype=torch.float32, device=q.device)
    _check(lib().scn_attn_fwd(SCN_TYPE[dtype], n, batch, pr, d, hq, hk, _ref(vq), _ref(vk),
                              _ref(vv), scale, l, r, sinks, _ref(vo), lse.data_ptr(),
                              _raw_stream(dev)), "scn_attn_fwd")
    return o, lse


def attn_bwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor,
             lse: torch.Tensor, do: torch.Tensor, ranges: torch.Tensor,
             left: Optional[int] = None, right: Optional[int] = None, sinks: int = 0,
             scale: Optional[float] = None, out=(None, None, None),
             ws: Optional[torch.Tensor] = None):
    """Gradients of ``attn_fwd`` (``scn_attn_bwd``): a dict with dq, dk and dv,
    in ``out`` where given (apart from the inputs).  Rows outside every range are
    not written, as in ``attn_fwd``."""
    dtype, dev, n, hq, hk, d, vq, vk, vv = _qkv(q, k, v)
    batch, pr, scale, l, r = _attn_args(ranges, dev, left, right, sinks, scale, d)
    vo = _rows(o, dtype, dev, (n, hq, d), "o")
    vg = _rows(do, dtype, dev, (n, hq, d), "do")
    pl = _vector(lse, torch.float32, dev, (hq, n), "lse")
    dq, wq = _out_rows(out[0], q, (n, hq, d), "out[0]")
    dk, wk = _out_rows(out[1], q, (n, hk, d), "out[1]")
    dv, wv = _out_rows(out[2], q, (n, hk, d), "out[2]")
    if ws is None:
        ws = _bytes(lib().scn_attn_bwd_workspace_bytes(n, batch, d, hq, hk, l, sinks), q.device)
    _check(lib().scn_attn_bwd(
        SCN_TYPE[dtype], n, batch, pr, d, hq, hk, _ref(vq), _ref(vk), _ref(vv), _ref(vo), pl,
        _ref(vg), scale, l, r, sinks, _ref(wq), _ref(wk), _ref(wv), ws.data_ptr(), ws.numel(),
        _raw_stream(dev)), "scn_attn_bwd")
    return {"dq": dq, "dk": dk, "dv": dv}


def attn_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor,
              v_cache: torch.Tensor, length: torch.Tensor, left: Optional[int] = None,
              sinks: int = 0, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
              ws: Optional[torch.Tensor] = None):
    """Attention of one new token of each stream (``scn_attn_step``).  q
    [streams, Hq, D], k and v [streams, Hk, D]; the caches [streams, capacity,
    Hk, D] (capacity > sinks; the rows past the sinks are a ring); length int32
    [streams], the tokens written before.  Writes the new keys and values to the
    caches and returns o [streams, Hq, D]; the caller advances length."""
    dtype, dev, b, hq, hk, d, vq, vk, vv = _qkv(q, k, v)
    cap = k_cache.shape[1] if isinstance(k_cache, torch.Tensor) and k_cache.dim() == 4 else 0
    ck = _cache(k_cache, dtype, dev, (b, cap, hk, d), "k_cache")
    cv = _cache(v_cache, dtype, dev, (b, cap, hk, d), "v_cache")
    pl = _vector(length, torch.int32, dev, (b,), "length")
    if not 0 <= sinks < cap:
        raise ValueError(f"sinks must lie in [0, capacity = {cap}), got {sinks}")
    l = _bound(left, "left")
    o, vo = _out_rows(out, q, (b, hq, d), "out")
    if ws is None:
        n = lib().scn_attn_step_workspace_bytes(SCN_TYPE[dtype], b, cap, d, hq, hk, l, sinks)
        ws = _bytes(n, q.device) if n else None
    _check(lib().scn_attn_step(
        SCN_TYPE[dtype], b, cap, d, hq, hk, _ref(vq), _ref(vk), _ref(vv), _ref(ck), _ref(cv), pl,
        d ** -0.5 if scale is None else scale, l, sinks, _ref(vo),
        None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(),
        _raw_stream(dev)), "scn_attn_step")
    return o


@functools.lru_cache(maxsize=4096)
def _sized(name: str, *sizes) -> int:
    """Workspace bytes of a call, a function of its sizes."""
    return getattr(lib(), name)(*sizes)


def _cross(q, k, v, q_ranges, k_ranges, scale):
    shape, dtype, dev = _first(q, "q")
    n, hq, d = shape
    m, hk = (k.shape[0], k.shape[1]) if isinstance(k, torch.Tensor) and k.dim() == 3 else (0, 0)
    vq = _rows(q, dtype, dev, shape, "q")
    vk = _rows(k, dtype, dev, (m, hk, d), "k")
    vv = _rows(v, dtype, dev, (m, hk, d), "v")
    if hk < 1 or hq % hk:
        raise ValueError(f"{hq} query heads cannot share {hk} key heads evenly")
    batch = q_ranges.shape[0] - 1 if isinstance(q_ranges, torch.Tensor) and q_ranges.dim() == 1 else 0
    if batch < 1:
        raise ValueError("q_ranges must hold at least two bounds")
    pq = _vector(q_ranges, torch.int32, dev, (batch + 1,), "q_ranges")
    pk = _vector(k_ranges, torch.int32, dev, (batch + 1,), "k_ranges")
    if pq is None or pk is None:
        raise TypeError("k_ranges must be a CUDA (HIP) tensor")
    return (dtype, dev, n, m, batch, pq, pk, d, hq, hk, vq, vk, vv,
            d ** -0.5 if scale is None else scale)


def cross_attn_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_ranges: torch.Tensor,
                   k_ranges: torch.Tensor, scale: Optional[float] = None,
                   out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """Attention of each sample's rows to the same sample's states
    (``scn_cross_attn_fwd``).  q [n, Hq, D], k and v [m, Hk, D], float32 or
    bfloat16, any row and head strides; the ranges int32 [batch + 1] as
    ``site_ranges`` gives, of q's rows and of the states.  scale is D ** -0.5 unless
    given.  Returns (o [n, Hq, D], lse float32 [Hq, n]); rows of samples without
    states get 0 and -inf, and rows outside every range are not written.  ``out``
    may not overlap q, k or v.  Streams whose states stay take their newest rows
    with ranges 0, 1, 2, .."""
    dtype, dev, n, m, batch, pq, pk, d, hq, hk, vq, vk, vv, scale = _cross(
        q, k, v, q_ranges, k_ranges, scale)
    o, vo = _out_rows(out, q, (n, hq, d), "out")
    lse = torch.empty((hq, n), dtype=torch.float32, device=q.device)
    if ws is None:
        need = _sized("scn_cross_attn_fwd_workspace_bytes", SCN_TYPE[dtype], n, m, batch, d, hq, hk)
        ws = _bytes(need, q.device) if need else None
    _check(lib().scn_cross_attn_fwd(
        SCN_TYPE[dtype], n, m, batch, pq, pk, d, hq, hk, _ref(vq), _ref(vk), _ref(vv), scale,
        _ref(vo), lse.data_ptr(), None if ws is None else ws.data_ptr(),
        0 if ws is None else ws.numel(), _raw_stream(dev)), "scn_cross_attn_fwd")
    return o, lse


def cross_attn_bwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor,
                   lse: torch.Tensor, do: torch.Tensor, q_ranges: torch.Tensor,
                   k_ranges: torch.Tensor, scale: Optional[float] = None,
                   out=(None, None, None), ws: Optional[torch.Tensor] = None):
    """Gradients of ``cross_attn_fwd`` (``scn_cross_attn_bwd``): a dict with dq, dk
    and dv, in ``out`` where given (apart from the inputs).  States of samples
    without rows of q, and rows of q without states, get 0; rows outside every range
    are not written."""
    dtype, dev, n, m, batch, pq, pk, d, hq, hk, vq, vk, vv, scale = _cross(
        q, k, v, q_ranges, k_ranges, scale)
    vo = _rows(o, dtype, dev, (n, hq, d), "o")
    vg = _rows(do, dtype, dev, (n, hq, d), "do")
    pl = _vector(lse, torch.float32, dev, (hq, n), "lse")
    dq, wq = _out_rows(out[0], q, (n, hq, d), "out[0]")
    dk, wk = _out_rows(out[1], q, (m, hk, d), "out[1]")
    dv, wv = _out_rows(out[2], q, (m, hk, d), "out[2]")
    if ws is None:
        ws = _bytes(_sized("scn_cross_attn_bwd_workspace_bytes", SCN_TYPE[dtype], n, m, batch, d,
                           hq, hk), q.device)
    _check(lib().scn_cross_attn_bwd(
        SCN_TYPE[dtype], n, m, batch, pq, pk, d, hq, hk, _ref(vq), _ref(vk), _ref(vv), _ref(vo), pl,
        _ref(vg), scale, _ref(wq), _ref(wk), _ref(wv), ws.data_ptr(), ws.numel(),
        _raw_stream(dev)), "scn_cross_attn_bwd")
    return {"dq": dq, "dk": dk, "dv": dv}


# ---------------------------------------------------------------------------
# norms around a block, clipping
# ---------------------------------------------------------------------------

def _matrix(t, dtype, device: int, shape, name: str):
    """ctypes view of a [rows, channels] tensor (any row stride with contiguous
    channels), or None."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.is_cuda and
            t.get_device() == device and t.shape == shape):
        _refuse_rows(t, dtype, device, shape, name)
    row, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise ValueError(f"{name} must have contiguous channels")
    return _Rows(t.data_ptr(), row if shape[0] > 1 else 0)


def _out_matrix(t, dtype, device, shape, name: str):
    """(result, its view), allocated here unless given; a given result's rows must
    not overlap."""
    if t is None:
        t = torch.empty(shape, dtype=dtype, device=device)
        return t, _Rows(t.data_ptr(), shape[1])
    v = _matrix(t, dtype, device.index, shape, name)
    if shape[0] > 1 and v.row < shape[1]:
        raise ValueError(f"{name} must not be expanded")
    return t, v


def _block(x, f, z, wf, wh, h):
    """The call's types, sizes and views; h: whose type the block's rows have without f."""
    for t, name in ((x, "x"), (f if f is not None else h if h is not None else x, "f")):
        if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in SCN_TYPE:
            _refuse_rows(t, None, -1, (), name)
        if t.dim() != 2:
            raise ValueError(f"{name} must have two dimensions, got {tuple(t.shape)}")
        typ = t.dtype
    dev = x.get_device()
    if dev != torch.cuda.current_device():
        raise ValueError(f"x is on cuda:{dev}, which is not the current device")
    if x.dtype == torch.bfloat16 and typ == torch.float32:
        raise TypeError("a residual of bfloat16 beside rows of float32")
    shape = tuple(x.shape)
    return (typ, dev, shape, _matrix(x, x.dtype, dev, shape, "x"), _matrix(f, typ, dev, shape, "f"),
            _matrix(z, typ, dev, shape, "z"), _vector(wf, torch.float32, dev, (shape[1],), "wf"),
            _vector(wh, torch.float32, dev, (shape[1],), "wh"))


def block_norm_fwd(x: torch.Tensor, f: Optional[torch.Tensor], z: Optional[torch.Tensor],
                   wf: Optional[torch.Tensor], wh: Optional[torch.Tensor], alpha: float = 1.0,
                   eps: float = 1e-6, need=("y", "h"), out=(None, None)):
    """A block's residual, gate and norms in one pass (``scn_block_norm_fwd``):
    y = alpha x + sigmoid(z) wf n(f) and h = wh n(y), n(t) = t / sqrt(mean t^2 +
    eps) over each row.  x [n, C] is the residual, float32 or bfloat16; f [n, C] the
    block's result (None: y = alpha x) and z [n, C] its gate's logits (None: no gate),
    of one type, bfloat16 beside a float32 residual too; any row strides.  wf, wh
    float32 [C] or None.  Returns (y, h), None where not in ``need`` (y of x's type, h
    of f's, or of out[1]'s or x's without f), in ``out`` where given (y may be x, h may
    be f or z)."""
    typ, dev, shape, vx, vf, vz, pf, ph = _block(x, f, z, wf, wh, out[1])
    y, vy = _out_matrix(out[0], x.dtype, x.device, shape, "out[0]") if "y" in need else (None, None)
    h, vh = _out_matrix(out[1], typ, x.device, shape, "out[1]") if "h" in need else (None, None)
    _check(lib().scn_block_norm_fwd(
        SCN_TYPE[x.dtype], SCN_TYPE[typ], shape[0], shape[1], _ref(vx), _ref(vf), _ref(vz), pf, ph,
        alpha, eps, _ref(vy), _ref(vh), _raw_stream(dev)), "scn_block_norm_fwd")
    return y, h


def block_norm_bwd(x: torch.Tensor, f: Optional[torch.Tensor], z: Optional[torch.Tensor],
                   wf: Optional[torch.Tensor], wh: Optional[torch.Tensor],
                   dy: Optional[torch.Tensor], dh: Optional[torch.Tensor], alpha: float = 1.0,
                   eps: float = 1e-6, need=("dwf", "dwh"), out=(None, None, None),
                   ws: Optional[torch.Tensor] = None):
    """Gradients of ``block_norm_fwd`` (``scn_block_norm_bwd``) for given dy (None:
    y has no other use than h) and dh (None: no h): a dict with dx, df and dz (with f
    and z alone; in ``out`` where given: dx may be dy, df and dz may be dh, f or z) and
    the requested ones of dwf, dwh."""
    typ, dev, shape, vx, vf, vz, pf, ph = _block(x, f, z, wf, wh, dh)
    vgy = _matrix(dy, x.dtype, dev, shape, "dy")
    vgh = _matrix(dh, typ, dev, shape, "dh")
    res, vdf, vdz = {}, None, None
    res["dx"], vdx = _out_matrix(out[0], x.dtype, x.device, shape, "out[0]")
    if f is not None:
        res["df"], vdf = _out_matrix(out[1], typ, x.device, shape, "out[1]")
    if z is not None:
        res["dz"], vdz = _out_matrix(out[2], typ, x.device, shape, "out[2]")
    pw = {}
    for name in ("dwf", "dwh"):
        if name in need and (name == "dwh" or f is not None):
            res[name] = torch.empty(shape[1], dtype=torch.float32, device=x.device)
            pw[name] = res[name].data_ptr()
    if ws is None:
        ws = _bytes(_sized("scn_block_norm_bwd_workspace_bytes", *shape) if pw else 0, x.device)
    _check(lib().scn_block_norm_bwd(
        SCN_TYPE[x.dtype], SCN_TYPE[typ], shape[0], shape[1], _ref(vx), _ref(vf), _ref(vz), pf, ph,
        alpha, eps, _ref(vgy), _ref(vgh), _ref(vdx), _ref(vdf), _ref(vdz), pw.get("dwf"),
        pw.get("dwh"), ws.data_ptr(), ws.numel(), _raw_stream(dev)), "scn_block_norm_bwd")
    return res


def _refuse_grad(t, dev: int, name: str):
    """What `clip_grads` does not take."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in SCN_TYPE:
        _refuse_rows(t, None, -1, (), name)
    if t.get_device() != dev:
        raise ValueError(f"{name} is on cuda:{t.get_device()}, which is not the current device")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def clip_grads(grads: Iterable[torch.Tensor], max_norm: float,
               out: Optional[Iterable[torch.Tensor]] = None,
               ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Clips gradients by the norm of all of them together (``scn_grad_clip``), in
    place or into ``out``: where the norm is finite and above ``max_norm`` (infinity:
    never) they are scaled by max_norm / norm.  Contiguous tensors, float32 and
    bfloat16 in any mix.  Returns the norm before, a float32 scalar on the device;
    nothing waits for it."""
    dev = torch.cuda.current_device()
    if not isinstance(grads, (list, tuple)):  # (a generator can be gone through once)
        grads = list(grads)
    if out is not None and not isinstance(out, (list, tuple)):
        out = list(out)
    try:  # whole lists at a time: many tensors are looked over with each call
        sizes = [t.numel() for t in grads]
        rows = [x for r in zip([t.data_ptr() for t in grads], sizes,
                               [SCN_TYPE[t.dtype] for t in grads]) for x in r]  # scn_tensor
        fine = all([t.get_device() == dev and t.is_contiguous() for t in grads])
    except (AttributeError, KeyError):
        fine = False
    if not fine:
        for i, t in enumerate(grads):
            _refuse_grad(t, dev, f"grads[{i}]")
    n, outs = len(sizes), None
    if out is not None:
        if len(out) != n:
            raise ValueError(f"out must hold {n} tensors, got {len(out)}")
        for i, (o, t) in enumerate(zip(out, grads)):
            if not (isinstance(o, torch.Tensor) and o.dtype == t.dtype and o.shape == t.shape and
                    o.get_device() == dev and o.is_contiguous()):
                _dev_tensor(o, t.dtype, t.shape, f"out[{i}]")
                raise TypeError(f"out[{i}] must be on cuda:{dev}, got {o.device}")
        outs = array("Q", [o.data_ptr() for o in out])
    rows = array("q", rows)
    device = torch.device("cuda", dev)
    norm = torch.empty((), dtype=torch.float32, device=device)
    if ws is None:
        need = lib().scn_grad_clip_workspace_bytes(n, sum(sizes))
        ws = _bytes(need, device) if need else None
    _check(lib().scn_grad_clip(
        n, rows.buffer_info()[0], None if outs is None else outs.buffer_info()[0], max_norm,
        norm.data_ptr(), None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(),
        _raw_stream(dev)), "scn_grad_clip")
    return norm


def version() -> str:
    return lib().scn_version().decode()


# Every callback pair ever installed stays alive for the life of the process:
# a rulebook built under a pair frees its memory through it, also after the
# pair has been replaced.
_hooks_kept = []


def build_chain(coords: torch.Tensor, grid, layers, lattice: str = "cubic") -> list:
    """Rulebooks of a chain of layers (``scn_rulebook_build_chain``): layer 0
    from ``coords`` on ``grid``, each later layer from the previous layer's
    active outputs; ``layers`` is a sequence of (filter, stride).  The chain
    waits for the device twice in all."""
    n = int(coords.shape[0]) if coords.dim() == 2 else -1
    _dev_tensor(coords, torch.int32, (n, 4), "coords")
    if lattice not in LATTICES:
        raise ValueError(f"lattice must be one of {sorted(LATTICES)}, got {lattice!r}")
    nl = len(layers)
    g = np.ascontiguousarray(np.asarray(grid, dtype=np.int64).reshape(4))
    fs = np.ascontiguousarray([int(f) for f, _ in layers], dtype=np.int32)
    ss = np.ascontiguousarray([int(s) for _, s in layers], dtype=np.int32)
    hs = (ctypes.c_void_p * max(nl, 1))()
    _check(lib().scn_rulebook_build_chain(
        _ptr(coords), n, g.ctypes.data_as(ctypes.c_void_p), LATTICES[lattice], nl,
        fs.ctypes.data_as(ctypes.c_void_p), ss.ctypes.data_as(ctypes.c_void_p),
        ctypes.c_void_p(_stream()), hs), "scn_rulebook_build_chain")
    return [Rulebook._from_handle(ctypes.c_void_p(hs[i]), coords.device) for i in range(nl)]


def set_dense_forward(min_rows: int = -1, min_offsets: int = -1) -> None:
    """Stride-1 rulebooks built from now on carry the dense forward view when
    they have at least ``min_rows`` outputs and ``min_offsets`` offsets
    (``scn_set_dense_forward``; negative values restore the defaults)."""
    _check(lib().scn_set_dense_forward(int(min_rows), int(min_offsets)), "scn_set_dense_forward")


def set_allocator(alloc=None, free=None) -> None:
    """Route the library's own device allocations through alloc(bytes, stream)
    -> pointer and free(pointer, stream) (``scn_set_allocator``).  ``"torch"``
    installs PyTorch's caching allocator; no argument restores the library's
    default pool."""
    if alloc == "torch":
        def alloc(nbytes, stream):
            return torch.cuda.caching_allocator_alloc(int(nbytes), stream=int(stream))

        def free(ptr, stream):
            torch.cuda.caching_allocator_delete(int(ptr))
    if alloc is None or free is None:
        lib().scn_set_allocator(_ALLOC_FN(), _FREE_FN(), None)
        return

    def c_alloc(nbytes, stream, ctx):
        try:
            return int(alloc(nbytes, stream or 0)) or None
        except Exception:  # the library reports SCN_ERR_NOMEM
            return None

    def c_free(ptr, stream, ctx):
        try:
            free(ptr, stream or 0)
        except Exception:
            pass

    hooks = (_ALLOC_FN(c_alloc), _FREE_FN(c_free))
    _hooks_kept.append(hooks)
    lib().scn_set_allocator(hooks[0], hooks[1], None)
