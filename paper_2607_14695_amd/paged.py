"""Python binding of the backbone operators: rotary positions over several axes, the paged K/V cache and the
attention of a chunk of new tokens over it (include/reflex.h, "Backbone operators").

Argument marshalling only, as in ``reflex.py``: every operator runs in the library's HIP kernels on the caller's
current stream of the tensors' device, and nothing waits for the GPU.  The operators record no gradients: a tensor
that needs one or carries a tangent is refused, by calls and as pages of a cache (``Rotary.apply(..., inverse=True)``
is the rotation's gradient).
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Tuple

import torch
from torch.autograd import forward_ad

from .reflex import (DTYPE_BF16, DTYPE_F32, STORE_BF16, STORE_F32, STORE_FP8, STORE_INT8, LADDERS, PagedBatchC,
                     PagedCacheC, RotaryC, RowsC, _check, load_library)

_DTYPES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}
_STORES = {torch.float32: STORE_F32, torch.bfloat16: STORE_BF16, torch.float8_e4m3fn: STORE_FP8,
           torch.int8: STORE_INT8}
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None


def _int32(x: int, what: str) -> int:
    """ctypes would cut an integer to its low 32 bits."""
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{what} {x} does not fit 32 bits")
    return x


def _dual_level() -> bool:
    """Whether forward-mode differentiation is on (if torch does not say, every tensor is asked)."""
    return getattr(forward_ad, "_current_level", 0) >= 0


def _no_gradient(x: torch.Tensor, what: str) -> None:
    """Refuse a tensor of which a gradient, or a tangent of forward-mode differentiation, would be dropped."""
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what} needs a gradient, which these operators do not record")
    if _dual_level() and forward_ad.unpack_dual(x).tangent is not None:
        raise ValueError(f"{what} carries a tangent, and these operators compute no gradient of either mode")


def _rows(x: torch.Tensor, n: int, heads: int, head_dim: int, device: torch.device, what: str) -> RowsC:
    """The C view of [n][heads][head_dim]; a dimension of one element may have any stride."""
    if x.shape != (n, heads, head_dim):
        raise ValueError(f"{what} is [{n}, {heads}, {head_dim}], got {tuple(x.shape)}")
    if x.device != device:
        raise ValueError(f"{what} is on {x.device}, not on {device}")
    if x.requires_grad or _dual_level():
        _no_gradient(x, what)
    rs, hs, es = x.stride()
    if es != 1:
        raise ValueError(f"{what} needs contiguous heads")
    return RowsC(x.data_ptr(), rs if n > 1 else 0, hs if heads > 1 else 0)


def _dtype(t: torch.dtype) -> int:
    d = _DTYPES.get(t)
    if d is None:
        raise ValueError(f"float32 or bfloat16 is computed in, not {t}")
    return d


def _index(x: torch.Tensor, shape: Sequence[int], dtype: torch.dtype, what: str, device=None) -> int:
    if x.dtype != dtype or x.shape != tuple(shape) or not x.is_contiguous():
        raise ValueError(f"{what} is a contiguous {dtype} tensor of shape {tuple(shape)}")
    if not x.is_cuda or (device is not None and x.device != device):
        raise ValueError(f"{what} is on {x.device}, not on {device or 'a GPU'}")
    return x.data_ptr()


def _call(device: torch.device, what: str, fn, *args) -> None:
    """fn(*args, stream) with the caller's current stream of `device`, that device current for the call."""
    idx = device.index
    if device.type != "cuda" or idx is None:
        raise ValueError(f"{what} runs on a GPU, not on {device}")
    if idx == torch.cuda.current_device():
        status = fn(*args, _raw_stream(idx))
    else:
        with torch.cuda.device(idx):
            status = fn(*args, _raw_stream(idx))
    if status:
        _check(status, what)


class Rotary:
    """A rotary plan: ``sections[a]`` pairs of dimensions follow axis a (default: one axis).

    ``ladder``: "shared" (one ladder of frequencies over all pairs) or "per_axis" (one for each axis)."""

    def __init__(self, head_dim: int, sections: Optional[Sequence[int]] = None, theta: float = 10000.0,
                 ladder: str = "shared"):
        if ladder not in LADDERS:
            raise ValueError(f"unknown ladder {ladder!r}")
        _int32(head_dim, "head_dim")
        sections = [head_dim // 2] if sections is None else [_int32(int(s), "sections:") for s in sections]
        self.lib = load_library()
        self.head_dim, self.sections, self.theta, self.ladder = head_dim, sections, theta, ladder
        self.c = RotaryC()
        arr = (ctypes.c_int32 * max(1, len(sections)))(*sections)
        _check(self.lib.reflex_rotary_init(ctypes.byref(self.c), head_dim, len(sections), arr, theta,
                                           LADDERS[ladder]), "reflex_rotary_init")
        self._ref = ctypes.byref(self.c)

    def _positions(self, positions: torch.Tensor, n: int, device: torch.device) -> Tuple[int, int]:
        """(pointer, stride between axes); [n] positions hold for every axis."""
        shape = (n,) if positions.dim() == 1 else (len(self.sections), n)
        p = _index(positions, shape, torch.int64, "positions", device)
        return p, (n if positions.dim() == 2 else 0)

    def apply(self, x: torch.Tensor, positions: torch.Tensor, inverse: bool = False,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [rows, heads, head_dim] rotated by ``positions`` (int64 [rows], or [axes, rows]).  ``out`` may be x."""
        if x.dim() != 3:
            raise ValueError(f"x is [rows, heads, head_dim], got {tuple(x.shape)}")
        n, heads, dh = x.shape
        device = x.device
        xr = _rows(x, n, heads, self.head_dim, device, "x")
        if out is None:
            out = torch.empty((n, heads, dh), dtype=x.dtype, device=device)
            yr = RowsC(out.data_ptr(), heads * dh, dh)
        else:
            if out.dtype != x.dtype:
                raise ValueError("out has x's type")
            yr = _rows(out, n, heads, dh, device, "out")
        p, ps = self._positions(positions, n, device)
        if heads:
            _call(device, "reflex_rotary_apply", self.lib.reflex_rotary_apply, self._ref, p, ps, ctypes.byref(xr),
                  ctypes.byref(yr), n, heads, _dtype(x.dtype), int(inverse))
        return out


class PagedBatch:
    """Which tokens a call is about: ``cu_rows`` [n + 1], ``lengths`` [n] and ``page_table`` [n, pages], contiguous
    int32 on the GPU, read there at every call (and at every replay of a captured one).  ``max_length``: the length
    that the longest sequence is expected to reach, which sizes the launches; longer ones stay correct."""

    def __init__(self, cu_rows: torch.Tensor, lengths: torch.Tensor, page_table: torch.Tensor, max_length: int = 0):
        if lengths.dim() != 1 or page_table.dim() != 2:
            raise ValueError("lengths is [sequences] and page_table [sequences, pages]")
        _int32(max_length, "max_length")
        n = lengths.shape[0]
        self.device = lengths.device
        self.tensors = (cu_rows, lengths, page_table)
        self.c = PagedBatchC(_index(cu_rows, (n + 1,), torch.int32, "cu_rows", self.device),
                             _index(lengths, (n,), torch.int32, "lengths"),
                             _index(page_table, (n, page_table.shape[1]), torch.int32, "page_table", self.device),
                             n, page_table.shape[1], max_length, 0)
        self._ref = ctypes.byref(self.c)


class PagedCache:
    """A paged K/V cache over the caller's tensors: k, v [pages, kv heads, page size, head dim] in float32, bfloat16,
    float8_e4m3fn or int8, the last two with float32 k_scale, v_scale [pages, kv heads, page size]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        if k.dim() != 4 or k.dtype not in _STORES:
            raise ValueError("k is [pages, kv heads, page size, head dim] in float32, bfloat16, float8_e4m3fn or int8")
        self.lib = load_library()
        self.device = k.device
        pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        scaled = k.element_size() == 1
        if scaled != (k_scale is not None) or scaled != (v_scale is not None):
            raise ValueError("8-bit pages have scales, others none")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        for what, t in (("k", k), ("v", v), ("k_scale", k_scale), ("v_scale", v_scale)):
            if t is not None:
                with torch.enable_grad():  # (the cache outlives a no_grad block that it is made in)
                    _no_gradient(t, what)
        self.c = PagedCacheC(
            _index(k, k.shape, k.dtype, "k"), _index(v, k.shape, k.dtype, "v", k.device),
            _index(k_scale, k.shape[:3], torch.float32, "k_scale", k.device) if scaled else None,
            _index(v_scale, k.shape[:3], torch.float32, "v_scale", k.device) if scaled else None,
            pages, self.page_size, self.n_kv_heads, self.head_dim, _STORES[k.dtype], 0)
        self._ref = ctypes.byref(self.c)

    @classmethod
    def zeros(cls, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype = torch.bfloat16,
              device: str = "cuda:0") -> "PagedCache":
        """A cache over new zeroed tensors."""
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        size = torch.empty(0, dtype=dtype).element_size()
        kv = [torch.zeros(shape, dtype=torch.uint8 if size == 1 else dtype, device=device).view(dtype)
              for _ in range(2)]
        scales = [torch.zeros(shape[:3], dtype=torch.float32, device=device) for _ in range(2)] if size == 1 else []
        return cls(*kv, *scales)

    def _batch(self, batch: PagedBatch):
        if batch.device != self.device:
            raise ValueError(f"the batch is on {batch.device}, the cache on {self.device}")
        return batch._ref

    def write(self, batch: PagedBatch, k: torch.Tensor, v: torch.Tensor, rotary: Optional[Rotary] = None,
              positions: Optional[torch.Tensor] = None) -> None:
        """Write the batch's rows k, v [rows, kv heads, head dim] into their pages, the keys rotated first where a
        plan is given: by ``positions``, or by each token's index in its sequence.  Rows for the same slot (sequences
        that share the page) have to be equal."""
        n = k.shape[0]
        if v.dtype != k.dtype:
            raise ValueError("k and v have one type")
        kr = _rows(k, n, self.n_kv_heads, self.head_dim, self.device, "k")
        vr = _rows(v, n, self.n_kv_heads, self.head_dim, self.device, "v")
        p, ps = None, 0
        if positions is not None:
            if rotary is None:
                raise ValueError("positions need a rotary plan")
            p, ps = rotary._positions(positions, n, self.device)
        _call(self.device, "reflex_paged_write", self.lib.reflex_paged_write, self._ref, self._batch(batch),
              ctypes.byref(kr), ctypes.byref(vr), n, _dtype(k.dtype), None if rotary is None else rotary._ref, p, ps)

    def read(self, batch: PagedBatch, n_rows: int, dtype: torch.dtype = torch.bfloat16,
             out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """k, v [n_rows, kv heads, head dim] of the batch's rows; without ``out``, rows of no sequence are
        undefined."""
        if out is None:
            kv = torch.empty((2, n_rows, self.n_kv_heads, self.head_dim), dtype=dtype, device=self.device)
            out = (kv[0], kv[1])
        k, v = out
        if k.dtype != v.dtype:
            raise ValueError("out is two tensors of one type")
        kr = _rows(k, n_rows, self.n_kv_heads, self.head_dim, self.device, "k")
        vr = _rows(v, n_rows, self.n_kv_heads, self.head_dim, self.device, "v")
        _call(self.device, "reflex_paged_read", self.lib.reflex_paged_read, self._ref, self._batch(batch),
              ctypes.byref(kr), ctypes.byref(vr), n_rows, _dtype(k.dtype))
        return out

    def attend(self, batch: PagedBatch, q: torch.Tensor, causal: bool = True, window: int = 0,
               scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of the batch's rows q [rows, heads, head dim] over the pages of their sequences, which hold
        the rows' own keys and values.  Scores are scaled by ``scale`` (default head_dim ** -0.5).  Without
        ``out``, rows of no sequence are undefined.  The workspace comes from torch's allocator, on the current
        stream."""
        if q.dim() != 3:
            raise ValueError(f"q is [rows, heads, head_dim], got {tuple(q.shape)}")
        n, heads, dh = q.shape
        dt = _dtype(q.dtype)
        _int32(window, "window")
        qr = _rows(q, n, heads, self.head_dim, self.device, "q")
        if out is None:
            out = torch.empty((n, heads, dh), dtype=q.dtype, device=self.device)
            yr = RowsC(out.data_ptr(), heads * dh, dh)
        else:
            if out.dtype != q.dtype:
                raise ValueError("out has q's type")
            yr = _rows(out, n, heads, dh, self.device, "out")
        ref = self._batch(batch)
        need = ctypes.c_size_t(0)
        status = self.lib.reflex_paged_attention_workspace(self._ref, ref, n, heads, dt, ctypes.byref(need))
        if status:
            _check(status, "reflex_paged_attention_workspace")
        nb = need.value
        ws = torch.empty(nb, dtype=torch.uint8, device=self.device) if nb else None
        _call(self.device, "reflex_paged_attention", self.lib.reflex_paged_attention, self._ref, ref,
              ctypes.byref(qr), ctypes.byref(yr), n, heads, dt, self.head_dim ** -0.5 if scale is None else scale,
              int(causal), window, ws.data_ptr() if nb else None, nb)
        return out
