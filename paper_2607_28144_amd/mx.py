"""Thin torch-facing binding of the MXFP4 kernels (include/regenvc_mx.h):
argument marshalling only; every step runs in the HIP kernels of
libregenvc_attn.so on torch's current stream.

MXFP4: blocks of 32 values of four bits under a power-of-two scale byte.
Matrices (MxTensor) and caches (KvCache) hold codes and scales as uint8 device
tensors in the layouts of regenvc_mx.h; quantize/dequantize and append/values
convert.  Workspaces are torch allocations on the current stream.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple, Union

import torch

from . import _lib
from .api import _DT, _desc, _fptr, _scale
from .dit import EPI, _rows, _vec

_stream = _lib.stream_of
_same_device = _lib.same_device


class MxTensor:
    """A matrix [rows, cols] in MXFP4: its codes and scales (uint8 device
    tensors in the layouts of regenvc_mx_bytes)."""

    __slots__ = ("codes", "scales", "rows", "cols")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int):
        nc, ns = mx_bytes(rows, cols)
        for name, t, n in (("codes", codes, nc), ("scales", scales, ns)):
            if t.device.type != "cuda" or t.dtype != torch.uint8 or not t.is_contiguous() or t.numel() != n:
                raise ValueError(f"{name} of a [{rows}, {cols}] matrix must be a contiguous uint8 device tensor of {n} bytes")
        if codes.device != scales.device:
            raise ValueError("codes and scales must be on one device")
        self.codes, self.scales, self.rows, self.cols = codes, scales, int(rows), int(cols)

    @property
    def shape(self) -> Tuple[int, int]:
        return self.rows, self.cols

    @property
    def device(self) -> torch.device:
        return self.codes.device


def mx_bytes(rows: int, cols: int) -> Tuple[int, int]:
    """Bytes of the codes and of the scales of a [rows, cols] matrix (regenvc_mx_bytes)."""
    nc, ns = ctypes.c_int64(), ctypes.c_int64()
    _lib.check(_lib.load().regenvc_mx_bytes(rows, cols, ctypes.byref(nc), ctypes.byref(ns)), "regenvc_mx_bytes")
    return nc.value, ns.value


def _float_dtype(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _DT:
        raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    return _DT[t.dtype]


def quantize(x: torch.Tensor, out: Optional[MxTensor] = None) -> MxTensor:
    """x (bf16 or float32 [rows, cols], unit column stride) in MXFP4 (regenvc_mx_quantize)."""
    dt = _float_dtype(x, "x")
    ldx = _rows(x, "x", x.dtype)
    rows, cols = x.shape
    if out is None:
        nc, ns = mx_bytes(rows, cols)
        out = MxTensor(torch.empty(nc, dtype=torch.uint8, device=x.device),
                       torch.empty(ns, dtype=torch.uint8, device=x.device), rows, cols)
    elif out.shape != (rows, cols):
        raise ValueError(f"out is {out.shape}, x {tuple(x.shape)}")
    _same_device(x.device, out=out.codes)
    with _lib.on_device(x.device):
        st = _lib.load().regenvc_mx_quantize(x.data_ptr(), dt, ldx, out.codes.data_ptr(), out.scales.data_ptr(), rows,
                                             cols, _stream(x.device))
    _lib.check(st, "regenvc_mx_quantize")
    return out


def dequantize(m: MxTensor, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values of an MXFP4 matrix as float32 or bf16 (regenvc_mx_dequantize)."""
    if out is None:
        out = torch.empty(m.shape, dtype=dtype, device=m.device)
    if tuple(out.shape) != m.shape:
        raise ValueError(f"out is {tuple(out.shape)}, the matrix {m.shape}")
    dt = _float_dtype(out, "out")
    ldo = _rows(out, "out", out.dtype)
    _same_device(m.device, out=out)
    with _lib.on_device(m.device):
        st = _lib.load().regenvc_mx_dequantize(m.codes.data_ptr(), m.scales.data_ptr(), out.data_ptr(), dt, ldo, m.rows,
                                               m.cols, _stream(m.device))
    _lib.check(st, "regenvc_mx_dequantize")
    return out


_NEED = {}  # (device index, shape, epilogue, quantized) -> least and total workspace bytes of a linear layer


def linear_workspace_bytes(M: int, N: int, K: int, epilogue: str, quantized: bool, device) -> Tuple[int, int]:
    """Workspace bytes that a linear layer must have and can use (regenvc_mx_linear_workspace)."""
    idx = _lib.device_index(device)
    key = (idx, M, N, K, epilogue, quantized)
    need = _NEED.get(key)
    if need is None:
        least, total = ctypes.c_int64(), ctypes.c_int64()
        st = _lib.load().regenvc_mx_linear_workspace(M, N, K, EPI[epilogue], int(quantized), _lib.compute_units(device),
                                                     ctypes.byref(least), ctypes.byref(total))
        # a shape the call itself refuses: let it say so
        need = (least.value, total.value) if st == _lib.OK else (0, 0)
        if len(_NEED) >= 4096:
            _NEED.clear()
        _NEED[key] = need
    return need


def linear_fwd(a: Union[torch.Tensor, MxTensor], w: MxTensor, bias: Optional[torch.Tensor] = None,
               epilogue: str = "bias", gate: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y = a w^T (+ bias) with both operands in MXFP4 and the epilogues of
    dit.linear_fwd (regenvc_mx_linear_fwd).  a: bf16 [M, K], brought to MXFP4
    by the call, or an MxTensor (of activations that several layers read)."""
    M, K = a.shape
    N = w.rows
    if w.cols != K:
        raise ValueError(f"w is {w.shape}, a {tuple(a.shape)}")
    quantized = isinstance(a, MxTensor)
    lda = 0 if quantized else _rows(a, "a", torch.bfloat16)
    epi = EPI[epilogue]
    if out is None:
        if epi == 2:
            raise ValueError("the gated-residual epilogue needs out (the float32 residual stream)")
        out = torch.empty((M, N), dtype=torch.bfloat16, device=a.device)
    elif tuple(out.shape) != (M, N):
        raise ValueError(f"out is {tuple(out.shape)}, y {(M, N)}")
    ldo = _rows(out, "out", torch.float32 if epi == 2 else torch.bfloat16)
    bp, gp = _vec(bias, "bias", torch.bfloat16, N), _vec(gate, "gate", torch.float32, N)
    _same_device(a.device, w=w.codes, bias=bias, gate=gate, out=out)
    least, total = linear_workspace_bytes(M, N, K, epilogue, quantized, a.device)
    with _lib.on_device(a.device):
        ws = _lib.split_workspace(total, a.device)
        if ws is None and least > 0:  # without the partial sums of a split of K
            ws = torch.empty(least, dtype=torch.uint8, device=a.device)
        st = _lib.load().regenvc_mx_linear_fwd(
            None if quantized else a.data_ptr(), lda, a.codes.data_ptr() if quantized else None,
            a.scales.data_ptr() if quantized else None, w.codes.data_ptr(), w.scales.data_ptr(), bp, gp, out.data_ptr(),
            ldo, M, N, K, epi, ws.data_ptr() if ws is not None else None, ws.numel() if ws is not None else 0,
            _stream(a.device))
    _lib.check(st, "regenvc_mx_linear_fwd")
    return out


def _ints(t: Optional[torch.Tensor], name: str, n: int, device: torch.device) -> Optional[int]:
    if t is None:
        return None
    if t.device != device or t.dtype != torch.int32 or not t.is_contiguous() or tuple(t.shape) != (n,):
        raise ValueError(f"{name} must be a contiguous int32 tensor of {n} elements on {device}")
    return t.data_ptr()


class KvCache:
    """Keys and values of `batch` sequences, `heads` key heads of D channels
    and `capacity` places each, in MXFP4 (regenvc_mx_cache).  A new cache holds
    zeros.  The caller keeps the lengths."""

    def __init__(self, batch: int, capacity: int, heads: int, D: int, device="cuda"):
        if D not in (64, 128):
            raise ValueError(f"D={D} (64 or 128)")
        self.batch, self.capacity, self.heads, self.D = int(batch), int(capacity), int(heads), int(D)
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError(f"a cache lies in device memory, not on {self.device}")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        shape = (self.batch, self.heads, self.capacity)
        self.k_codes, self.v_codes = (torch.zeros(*shape, D // 2, dtype=torch.uint8, device=self.device) for _ in range(2))
        self.k_scales, self.v_scales = (torch.zeros(*shape, D // 32, dtype=torch.uint8, device=self.device)
                                        for _ in range(2))

    def _c(self) -> _lib.MxCache:
        return _lib.MxCache(self.k_codes.data_ptr(), self.k_scales.data_ptr(), self.v_codes.data_ptr(),
                            self.v_scales.data_ptr(), self.batch, self.capacity, self.heads, self.D)

    def append(self, k: torch.Tensor, v: torch.Tensor, start: Optional[torch.Tensor] = None,
               count: Optional[torch.Tensor] = None) -> None:
        """Tokens k, v (bf16 [batch, S, heads, D]) to places (start[b] + i) mod
        capacity, the first count[b] of each sequence (int32 device tensors;
        default 0 and S) (regenvc_mx_cache_append)."""
        S = k.shape[1]
        want = (self.batch, S, self.heads, self.D)
        if tuple(k.shape) != want or tuple(v.shape) != want:
            raise ValueError(f"k, v must be {list(want)}, got {tuple(k.shape)}, {tuple(v.shape)}")
        kd, vd = _desc(k, "k", torch.bfloat16), _desc(v, "v", torch.bfloat16)
        _same_device(self.device, k=k, v=v)
        sp, cp = _ints(start, "start", self.batch, self.device), _ints(count, "count", self.batch, self.device)
        c = self._c()
        with _lib.on_device(self.device):
            st = _lib.load().regenvc_mx_cache_append(ctypes.byref(c), ctypes.byref(kd), ctypes.byref(vd), S, sp, cp,
                                                     _stream(self.device))
        _lib.check(st, "regenvc_mx_cache_append")

    def values(self, dtype: torch.dtype = torch.float32) -> Tuple[torch.Tensor, torch.Tensor]:
        """The cache's keys and values as float32 or bf16 [batch, capacity,
        heads, D] (regenvc_mx_cache_values)."""
        k, v = (torch.empty((self.batch, self.capacity, self.heads, self.D), dtype=dtype, device=self.device)
                for _ in range(2))
        dt = _float_dtype(k, "dtype")
        c = self._c()
        with _lib.on_device(self.device):
            st = _lib.load().regenvc_mx_cache_values(ctypes.byref(c), k.data_ptr(), v.data_ptr(), dt, _stream(self.device))
        _lib.check(st, "regenvc_mx_cache_values")
        return k, v


_ATTN_NEED = {}  # (device index, shape) -> workspace bytes of a call


def _attn_need(B: int, H: int, heads: int, Sq: int, max_len: int, D: int, device: torch.device) -> int:
    key = (device.index, B, H, heads, Sq, max_len, D)
    need = _ATTN_NEED.get(key)
    if need is None:
        out = ctypes.c_int64()
        st = _lib.load().regenvc_mx_attn_cache_workspace(B, H, heads, Sq, max_len, D, _lib.compute_units(device), ctypes.byref(out))
        need = out.value if st == _lib.OK else 0  # a shape the call itself refuses: let it say so
        if len(_ATTN_NEED) >= 4096:
            _ATTN_NEED.clear()
        _ATTN_NEED[key] = need
    return need


def attn_cache_fwd(q: torch.Tensor, cache: KvCache, lens: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                   max_len: Optional[int] = None, out_dtype: torch.dtype = torch.bfloat16,
                   out: Optional[torch.Tensor] = None, return_lse: bool = True, lse_out: Optional[torch.Tensor] = None
                   ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Exact attention of q (bf16 [batch, Sq, H, D]; H a multiple of the
    cache's heads) over the first lens[b] places of each sequence (int32 device
    tensor; default max_len for all) (regenvc_mx_attn_cache_fwd).  max_len
    (default: the capacity) is the length that the work is planned for.
    Returns (O, LSE or None); a sequence without a place gives 0 and -inf."""
    if q.dim() != 4:
        raise ValueError(f"q must be [batch, Sq, H, D], got {tuple(q.shape)}")
    B, Sq, H, D = q.shape
    if B != cache.batch or D != cache.D:
        raise ValueError(f"q is {tuple(q.shape)}, the cache holds {cache.batch} sequences of D={cache.D}")
    if out is None:
        out = torch.empty((B, Sq, H, D), dtype=out_dtype, device=q.device)
    elif tuple(out.shape) != (B, Sq, H, D):
        raise ValueError(f"out is {tuple(out.shape)}, q {tuple(q.shape)}")
    if lse_out is None and return_lse:
        lse_out = torch.empty((B, H, Sq), dtype=torch.float32, device=q.device)
    if out_dtype not in _DT:
        raise TypeError(f"out_dtype must be bfloat16 or float32, got {out_dtype}")
    qd, od = _desc(q, "q", torch.bfloat16), _desc(out, "out", out_dtype)
    lp = _fptr(lse_out, "lse", (B, H, Sq))
    _same_device(cache.device, q=q, out=out, lse_out=lse_out)
    np = _ints(lens, "lens", B, cache.device)
    n = cache.capacity if max_len is None else int(max_len)
    need = _attn_need(B, H, cache.heads, Sq, n, D, cache.device)
    c = cache._c()
    with _lib.on_device(cache.device):
        ws = torch.empty(need, dtype=torch.uint8, device=cache.device) if need > 0 else None
        st = _lib.load().regenvc_mx_attn_cache_fwd(
            ctypes.byref(qd), ctypes.byref(c), np, n, ctypes.byref(od), _DT[out_dtype], lp, B, H, Sq, _scale(scale, D),
            ws.data_ptr() if ws is not None else None, need, _stream(cache.device))
    _lib.check(st, "regenvc_mx_attn_cache_fwd")
    return out, lse_out
