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
from .dit import EPI


class MxTensor:
    """A matrix [rows, cols] in MXFP4: its codes and scales (uint8 device
    tensors in the layouts of regenvc_mx_bytes)."""

    __slots__ = ("codes", "scales", "rows", "cols")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int):
        nc, ns = mx_bytes(rows, cols)
        idx = _lib.index_of(codes, "codes")
        _lib.vector(codes, "codes", torch.uint8, nc, idx)
        _lib.vector(scales, "scales", torch.uint8, ns, idx)
        self.codes, self.scales, self.rows, self.cols = codes, scales, int(rows), int(cols)

    @property
    def shape(self) -> Tuple[int, int]:
        return self.rows, self.cols

    @property
    def device(self) -> torch.device:
        return self.codes.device


def mx_bytes(rows: int, cols: int) -> Tuple[int, int]:
    """Bytes of the codes and of the scales of a [rows, cols] matrix (regenvc_mx_bytes)."""
    _lib.int32(rows=rows, cols=cols)
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
    idx = _lib.index_of(x, "x")
    rows, cols = x.shape
    ldx = _lib.matrix(x, "x", x.dtype, rows, cols, idx)
    if out is None:
        nc, ns = mx_bytes(rows, cols)
        out = MxTensor(torch.empty(nc, dtype=torch.uint8, device=x.device),
                       torch.empty(ns, dtype=torch.uint8, device=x.device), rows, cols)
    elif out.shape != (rows, cols) or out.codes.get_device() != idx:
        raise ValueError(f"out is {out.shape} on {out.device}, x {tuple(x.shape)} on {x.device}")
    with _lib.on_device(idx):
        st = _lib.load().regenvc_mx_quantize(x.data_ptr(), dt, ldx, out.codes.data_ptr(), out.scales.data_ptr(), rows,
                                             cols, _lib.raw_stream(idx))
    _lib.check(st, "regenvc_mx_quantize")
    return out


def dequantize(m: MxTensor, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values of an MXFP4 matrix as float32 or bf16 (regenvc_mx_dequantize)."""
    if out is None:
        out = torch.empty(m.shape, dtype=dtype, device=m.device)
    dt = _float_dtype(out, "out")
    idx = m.codes.get_device()
    ldo = _lib.matrix(out, "out", out.dtype, m.rows, m.cols, idx)
    with _lib.on_device(idx):
        st = _lib.load().regenvc_mx_dequantize(m.codes.data_ptr(), m.scales.data_ptr(), out.data_ptr(), dt, ldo, m.rows,
                                               m.cols, _lib.raw_stream(idx))
    _lib.check(st, "regenvc_mx_dequantize")
    return out


_NEED = {}  # (shape, quantized) -> workspace bytes of a linear layer


def linear_workspace_bytes(M: int, N: int, K: int, quantized: bool) -> int:
    """Workspace bytes of a linear layer (regenvc_mx_linear_workspace)."""
    key = (M, N, K, quantized)
    need = _NEED.get(key)
    if need is None:
        _lib.int32(M=M, N=N, K=K)
        out = ctypes.c_int64()
        st = _lib.load().regenvc_mx_linear_workspace(M, N, K, int(quantized), ctypes.byref(out))
        need = out.value if st == _lib.OK else 0  # a shape the call itself refuses: let it say so
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
    idx = w.codes.get_device()
    if quantized:
        ac = a.codes
        if ac.get_device() != idx:
            raise ValueError(f"a is on {a.device}, w on {w.device}")
        a_ptr, lda, c_ptr, s_ptr = None, 0, ac.data_ptr(), a.scales.data_ptr()
    else:
        lda = _lib.matrix(a, "a", torch.bfloat16, M, K, idx)
        a_ptr, c_ptr, s_ptr = a.data_ptr(), None, None
    epi = EPI[epilogue]
    if out is not None:
        ldo = _lib.matrix(out, "out", torch.float32 if epi == 2 else torch.bfloat16, M, N, idx)
    elif epi == 2:
        raise ValueError("the gated-residual epilogue needs out (the float32 residual stream)")
    else:
        out, ldo = torch.empty(M, N, dtype=torch.bfloat16, device=a.device), N
    bp = _lib.vector(bias, "bias", torch.bfloat16, N, idx)
    gp = _lib.vector(gate, "gate", torch.float32, N, idx)
    need = linear_workspace_bytes(M, N, K, quantized)
    with _lib.on_device(idx):
        ws = torch.empty(need, dtype=torch.uint8, device=a.device) if need > 0 else None
        st = _lib.load().regenvc_mx_linear_fwd(
            a_ptr, lda, c_ptr, s_ptr, w.codes.data_ptr(), w.scales.data_ptr(), bp, gp, out.data_ptr(), ldo, M, N, K, epi,
            ws.data_ptr() if ws is not None else None, need, _lib.raw_stream(idx))
    _lib.check(st, "regenvc_mx_linear_fwd")
    return out


class KvCache:
    """Keys and values of `batch` sequences, `heads` key heads of D channels
    and `capacity` places each, in MXFP4 (regenvc_mx_cache).  A new cache holds
    zeros.  The caller keeps the lengths."""

    def __init__(self, batch: int, capacity: int, heads: int, D: int, device="cuda"):
        if D not in (64, 128):
            raise ValueError(f"D={D} (64 or 128)")
        _lib.int32(batch=batch, capacity=capacity, heads=heads)
        self.batch, self.capacity, self.heads, self.D = int(batch), int(capacity), int(heads), int(D)
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError(f"a cache lies in device memory, not on {self.device}")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        shape = (self.batch, self.heads, self.capacity)
        self._parts = tuple(torch.zeros(*shape, n, dtype=torch.uint8, device=self.device)
                            for n in (D // 2, D // 32, D // 2, D // 32))
        self._c = _lib.MxCache(*(t.data_ptr() for t in self._parts), self.batch, self.capacity, self.heads, self.D)

    # read-only: the addresses of the four tensors are in what the calls get
    k_codes = property(lambda self: self._parts[0])
    k_scales = property(lambda self: self._parts[1])
    v_codes = property(lambda self: self._parts[2])
    v_scales = property(lambda self: self._parts[3])

    def append(self, k: torch.Tensor, v: torch.Tensor, start: Optional[torch.Tensor] = None,
               count: Optional[torch.Tensor] = None) -> None:
        """Tokens k, v (bf16 [batch, S, heads, D]) to places (start[b] + i) mod
        capacity, the first count[b] of each sequence (int32 device tensors;
        default 0 and S) (regenvc_mx_cache_append)."""
        if k.dim() != 4 or v.shape != k.shape or k.shape[0] != self.batch or k.shape[2] != self.heads \
                or k.shape[3] != self.D:
            raise ValueError(f"k, v must be [{self.batch}, S, {self.heads}, {self.D}], got {tuple(k.shape)}, {tuple(v.shape)}")
        S = k.shape[1]
        if S >= 1 << 31:
            _lib.int32(S=S)
        idx = self.device.index
        kd, vd = _desc(k, "k", torch.bfloat16), _desc(v, "v", torch.bfloat16)
        if k.get_device() != idx or v.get_device() != idx:
            raise ValueError(f"k and v must be on {self.device}, got {k.device}, {v.device}")
        sp = _lib.vector(start, "start", torch.int32, self.batch, idx)
        cp = _lib.vector(count, "count", torch.int32, self.batch, idx)
        with _lib.on_device(idx):
            st = _lib.load().regenvc_mx_cache_append(ctypes.byref(self._c), ctypes.byref(kd), ctypes.byref(vd), S, sp, cp,
                                                     _lib.raw_stream(idx))
        _lib.check(st, "regenvc_mx_cache_append")

    def values(self, dtype: torch.dtype = torch.float32) -> Tuple[torch.Tensor, torch.Tensor]:
        """The cache's keys and values as float32 or bf16 [batch, capacity,
        heads, D] (regenvc_mx_cache_values)."""
        k, v = (torch.empty(self.batch, self.capacity, self.heads, self.D, dtype=dtype, device=self.device)
                for _ in range(2))
        dt = _float_dtype(k, "dtype")
        idx = self.device.index
        with _lib.on_device(idx):
            st = _lib.load().regenvc_mx_cache_values(ctypes.byref(self._c), k.data_ptr(), v.data_ptr(), dt,
                                                     _lib.raw_stream(idx))
        _lib.check(st, "regenvc_mx_cache_values")
        return k, v


_ATTN_NEED = {}  # (device index, shape) -> workspace bytes of a call


def _attn_need(B: int, H: int, heads: int, Sq: int, max_len: int, D: int, idx: int) -> int:
    key = (idx, B, H, heads, Sq, max_len, D)
    need = _ATTN_NEED.get(key)
    if need is None:
        _lib.int32(B=B, H=H, Sq=Sq, max_len=max_len)
        out = ctypes.c_int64()
        st = _lib.load().regenvc_mx_attn_cache_workspace(B, H, heads, Sq, max_len, D, _lib.compute_units(idx),
                                                         ctypes.byref(out))
        need = out.value if st == _lib.OK else 0  # a shape the call itself refuses: let it say so
        if len(_ATTN_NEED) >= 4096:
            _ATTN_NEED.clear()
        _ATTN_NEED[key] = need
    return need


def attn_cache_fwd(q: torch.Tensor, cache: KvCache, lens: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                   max_len: Optional[int] = None, out_dtype: torch.dtype = torch.bfloat16,
                   out: Optional[torch.Tensor] = None, return_lse: bool = True, lse_out: Optional[torch.Tensor] = None
                   ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Attention of q (bf16 [batch, Sq, H, D]; H a multiple of the cache's
    heads) over all of the first lens[b] places of each sequence (int32 device
    tensor; default max_len for all) (regenvc_mx_attn_cache_fwd).  Softmax
    weights multiply the values in bf16, whatever out_dtype is.  max_len
    (default: the capacity) is the length that the work is planned for.
    Returns (O, LSE or None); a sequence without a place gives 0 and -inf."""
    if q.dim() != 4:
        raise ValueError(f"q must be [batch, Sq, H, D], got {tuple(q.shape)}")
    B, Sq, H, D = q.shape
    if B != cache.batch or D != cache.D:
        raise ValueError(f"q is {tuple(q.shape)}, the cache holds {cache.batch} sequences of D={cache.D}")
    if out_dtype not in _DT:
        raise TypeError(f"out_dtype must be bfloat16 or float32, got {out_dtype}")
    idx, dev = cache.device.index, cache.device
    if out is None:
        out = torch.empty(B, Sq, H, D, dtype=out_dtype, device=dev)
        od = _lib.Tensor(out.data_ptr(), Sq * H * D, H * D, D)
    elif tuple(out.shape) != (B, Sq, H, D) or out.get_device() != idx:
        raise ValueError(f"out must be {(B, Sq, H, D)} on {dev}, got {tuple(out.shape)} on {out.device}")
    else:
        od = _desc(out, "out", out_dtype)
    qd = _desc(q, "q", torch.bfloat16)
    if q.get_device() != idx:
        raise ValueError(f"q is on {q.device}, the cache on {dev}")
    if lse_out is not None:
        lp = _fptr(lse_out, "lse", (B, H, Sq))
        if lse_out.get_device() != idx:
            raise ValueError(f"lse is on {lse_out.device}, the cache on {dev}")
    elif return_lse:
        lse_out = torch.empty(B, H, Sq, dtype=torch.float32, device=dev)
        lp = lse_out.data_ptr()
    else:
        lp = None
    np = _lib.vector(lens, "lens", torch.int32, B, idx)
    n = cache.capacity if max_len is None else int(max_len)
    need = _attn_need(B, H, cache.heads, Sq, n, D, idx)
    with _lib.on_device(idx):
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
        st = _lib.load().regenvc_mx_attn_cache_fwd(
            ctypes.byref(qd), ctypes.byref(cache._c), np, n, ctypes.byref(od), _DT[out_dtype], lp, B, H, Sq,
            _scale(scale, D), ws.data_ptr() if ws is not None else None, need, _lib.raw_stream(idx))
    _lib.check(st, "regenvc_mx_attn_cache_fwd")
    return out, lse_out
