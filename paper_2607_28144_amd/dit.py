"""Thin torch-facing binding of the diffusion-transformer block kernels
(include/regenvc_dit.h): argument marshalling only; every step runs in the
HIP kernels of libregenvc_attn.so on torch's current stream.

Tensors: activations are bf16 or (the residual stream) float32 [rows, C]
with unit column stride; linear weights bf16 [out, in] contiguous; biases
and normalization scales bf16 [n]; modulation vectors float32.
"""
from __future__ import annotations

import ctypes
from typing import Dict, NamedTuple, Optional, Tuple

import torch

from . import _lib

EPI = {"bias": 0, "bias_gelu": 1, "gated_residual": 2}


_stream = _lib.stream_of


def _rows(t: torch.Tensor, name: str, dtype: torch.dtype) -> int:
    if t.device.type != "cuda" or t.dtype != dtype or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a {dtype} device tensor [rows, cols] with unit column stride")
    return t.stride(0)


def _vec(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, n: int) -> Optional[int]:
    if t is None:
        return None
    if t.device.type != "cuda" or t.dtype != dtype or not t.is_contiguous() or t.numel() != n:
        raise ValueError(f"{name} must be a contiguous {dtype} device tensor of {n} elements")
    return t.data_ptr()


_N_CU = {}   # device index -> compute units
_NEED = {}   # (device index, shape, epilogue) -> workspace bytes of a linear layer


def linear_workspace_bytes(M: int, N: int, K: int, epilogue: str, device) -> int:
    """Workspace bytes of the split-K form of one linear layer on this device
    (regenvc_linear_workspace; host-only, 0 when it does not split)."""
    idx = torch.device(device).index
    idx = torch.cuda.current_device() if idx is None else idx
    need = _NEED.get((idx, M, N, K, epilogue))
    if need is None:
        if idx not in _N_CU:
            _N_CU[idx] = torch.cuda.get_device_properties(idx).multi_processor_count
        out = ctypes.c_int64()
        st = _lib.load().regenvc_linear_workspace(M, N, K, EPI[epilogue], _N_CU[idx], ctypes.byref(out))
        need = out.value if st == _lib.OK else 0  # a shape the call itself refuses: let it say so
        if len(_NEED) >= 4096:
            _NEED.clear()
        _NEED[(idx, M, N, K, epilogue)] = need
    return need


def linear_fwd(a: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, epilogue: str = "bias",
               gate: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y = a w^T (+ bias) with a fused epilogue (regenvc_linear_fwd_ws):
    'bias' -> bf16 out, 'bias_gelu' -> bf16 gelu_tanh(y), 'gated_residual' ->
    out (float32, required) += gate * y.  The workspace of the split-K form is
    a torch allocation on the current stream; without room for it K is not
    split."""
    M, K = a.shape
    N = w.shape[0]
    lda = _rows(a, "a", torch.bfloat16)
    if tuple(w.shape) != (N, K) or not w.is_contiguous() or w.dtype != torch.bfloat16:
        raise ValueError("w must be a contiguous bf16 [N, K] tensor")
    epi = EPI[epilogue]
    if out is None:
        if epi == 2:
            raise ValueError("the gated-residual epilogue needs out (the float32 residual stream)")
        out = torch.empty((M, N), dtype=torch.bfloat16, device=a.device)
    ldo = _rows(out, "out", torch.float32 if epi == 2 else torch.bfloat16)
    need = linear_workspace_bytes(M, N, K, epilogue, a.device)
    ws = _lib.split_workspace(need, a.device)
    st = _lib.load().regenvc_linear_fwd_ws(a.data_ptr(), lda, w.data_ptr(), _vec(bias, "bias", torch.bfloat16, N),
                                           _vec(gate, "gate", torch.float32, N), out.data_ptr(), ldo, M, N, K, epi,
                                           ws.data_ptr() if ws is not None else None, need if ws is not None else 0,
                                           _stream(a.device))
    _lib.check(st, "regenvc_linear_fwd_ws")
    return out


def layer_norm_fwd(x: torch.Tensor, shift=None, scale=None, w=None, b=None, eps: float = 1e-6,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """bf16 LN(x)(1 + scale) + shift (float32 shift/scale), or LN(x) w + b
    (bf16 w, b), of float32 rows x (regenvc_layer_norm_fwd)."""
    rows, C = x.shape
    ldx = _rows(x, "x", torch.float32)
    out = torch.empty((rows, C), dtype=torch.bfloat16, device=x.device) if out is None else out
    ldy = _rows(out, "out", torch.bfloat16)
    st = _lib.load().regenvc_layer_norm_fwd(
        x.data_ptr(), ldx, out.data_ptr(), ldy, _vec(shift, "shift", torch.float32, C),
        _vec(scale, "scale", torch.float32, C), _vec(w, "w", torch.bfloat16, C), _vec(b, "b", torch.bfloat16, C),
        rows, C, float(eps), _stream(x.device))
    _lib.check(st, "regenvc_layer_norm_fwd")
    return out


def rms_norm_fwd(x: torch.Tensor, w: torch.Tensor, eps: float = 1e-6,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """bf16 x / rms(x) w of bf16 rows (regenvc_rms_norm_fwd); out may be x."""
    rows, C = x.shape
    ldx = _rows(x, "x", torch.bfloat16)
    out = torch.empty_like(x) if out is None else out
    ldy = _rows(out, "out", torch.bfloat16)
    st = _lib.load().regenvc_rms_norm_fwd(x.data_ptr(), ldx, out.data_ptr(), ldy, _vec(w, "w", torch.bfloat16, C),
                                          rows, C, float(eps), _stream(x.device))
    _lib.check(st, "regenvc_rms_norm_fwd")
    return out


def modulation(w_mod: torch.Tensor, b_mod: torch.Tensor, e: torch.Tensor,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """float32 W_mod silu(e) + b_mod (regenvc_dit_modulation)."""
    rows, C = w_mod.shape
    out = torch.empty(rows, dtype=torch.float32, device=e.device) if out is None else out
    st = _lib.load().regenvc_dit_modulation(_vec(w_mod, "w_mod", torch.bfloat16, rows * C),
                                            _vec(b_mod, "b_mod", torch.bfloat16, rows),
                                            _vec(e, "e", torch.float32, C), _vec(out, "out", torch.float32, rows),
                                            rows, C, _stream(e.device))
    _lib.check(st, "regenvc_dit_modulation")
    return out


_NORM = {None: 0, "layer": 1, "rms": 2}
_ACT = {torch.bfloat16: _lib.BF16, torch.float32: _lib.F32}


def _norm(kind: Optional[str], eps: float, w, b, C: int, name: str, idx: int) -> _lib.Norm:
    if kind not in _NORM or (kind is None and name == "norm"):
        raise ValueError(f"{name}={kind!r} ('layer', 'rms'" + (" or None)" if name == "post" else ")"))
    return _lib.Norm(_NORM[kind], eps, _lib.vector(w, f"{name} w", torch.bfloat16, C, idx) if w is not None else None,
                     _lib.vector(b, f"{name} b", torch.bfloat16, C, idx) if b is not None else None)


def _row_vectors(groups: int, C: int, group_rows: int, idx: int, gate, scale, shift) -> _lib.RowVectors:
    """gate, scale, shift (or None): float32 [C], or [groups, C] with one row stride."""
    if groups == 1:  # [C] or [1, C]
        f32, vector = torch.float32, _lib.vector
        return _lib.RowVectors(vector(gate, "gate", f32, C, idx), vector(scale, "scale", f32, C, idx),
                               vector(shift, "shift", f32, C, idx), C, group_rows)
    ld = None
    ptrs = []
    for name, t in (("gate", gate), ("scale", scale), ("shift", shift)):
        if t is None:
            ptrs.append(None)
            continue
        step = _lib.matrix(t, name, torch.float32, groups, C, idx)
        if ld is not None and step != ld:
            raise ValueError("gate, scale and shift must have one row stride")
        ld = step
        ptrs.append(t.data_ptr())
    return _lib.RowVectors(ptrs[0], ptrs[1], ptrs[2], C if ld is None else ld, group_rows)


def _groups(rows: int, group_rows: int) -> Tuple[int, int]:
    """The sets of vectors of a call, and group_rows as the library gets it: any number from the rows on is one set."""
    if rows >= 1 << 31 or group_rows < -1:
        _lib.int32(rows=rows, group_rows=min(group_rows, rows))
    if group_rows >= rows:
        return 1, rows
    return -(-rows // group_rows) if group_rows > 0 else 1, group_rows


def residual_norm_fwd(x: torch.Tensor, y: torch.Tensor, norm: str = "layer", post: Optional[str] = None,
                      gate: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                      shift: Optional[torch.Tensor] = None, w: Optional[torch.Tensor] = None,
                      b: Optional[torch.Tensor] = None, post_w: Optional[torch.Tensor] = None,
                      post_b: Optional[torch.Tensor] = None, alpha: float = 1.0, eps: float = 1e-6,
                      group_rows: int = 0, out: Optional[torch.Tensor] = None,
                      h: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The seam between two branches (regenvc_residual_norm_fwd): x' = alpha x +
    gate N_post(y), h = N_pre(x') (1 + scale) + shift (or w, b).  x: float32
    [rows, C]; y: bf16 or float32; post, norm: 'layer' or 'rms' (post may be
    None); gate, scale, shift: float32 [C], or [groups, C] with a set for every
    group_rows rows.  out may be x.  Returns (x', h), h in y's type."""
    idx = _lib.index_of(x, "x")
    rows, C = x.shape
    act = y.dtype
    if act not in _ACT:
        raise ValueError(f"y must be bfloat16 or float32, got {act}")
    ldx, ldy = _lib.matrix(x, "x", torch.float32, rows, C, idx), _lib.matrix(y, "y", act, rows, C, idx)
    dev = x.device
    if out is None:
        out, ldo = torch.empty(rows, C, dtype=torch.float32, device=dev), C
    else:
        ldo = _lib.matrix(out, "out", torch.float32, rows, C, idx)
    if h is None:
        h, ldh = torch.empty(rows, C, dtype=act, device=dev), C
    else:
        ldh = _lib.matrix(h, "h", act, rows, C, idx)
    groups, group_rows = _groups(rows, group_rows)
    v = _row_vectors(groups, C, group_rows, idx, gate, scale, shift)
    np, nq = _norm(post, eps, post_w, post_b, C, "post", idx), _norm(norm, eps, w, b, C, "norm", idx)
    with _lib.on_device(idx):
        st = _lib.load().regenvc_residual_norm_fwd(
            x.data_ptr(), ldx, y.data_ptr(), ldy, _ACT[act], ctypes.byref(np), ctypes.byref(nq), ctypes.byref(v), alpha,
            out.data_ptr(), ldo, h.data_ptr(), ldh, rows, C, _lib.raw_stream(idx))
    _lib.check(st, "regenvc_residual_norm_fwd")
    return out, h


class ResidualNormGrads(NamedTuple):
    """Gradients of residual_norm_fwd; those of vectors that were not given are None."""
    dx: torch.Tensor
    dy: torch.Tensor
    dgate: Optional[torch.Tensor] = None
    dscale: Optional[torch.Tensor] = None
    dshift: Optional[torch.Tensor] = None
    dw: Optional[torch.Tensor] = None
    db: Optional[torch.Tensor] = None
    dpost_w: Optional[torch.Tensor] = None
    dpost_b: Optional[torch.Tensor] = None


_BWD_NEED = {}  # (device index, shape, sums) -> workspace bytes of a backward call


def _bwd_need(rows: int, C: int, group_rows: int, group_sums: int, row_sums: int, idx: int) -> int:
    key = (idx, rows, C, group_rows, group_sums, row_sums)
    need = _BWD_NEED.get(key)
    if need is None:
        out = ctypes.c_int64()
        st = _lib.load().regenvc_residual_norm_bwd_workspace(rows, C, group_rows, group_sums, row_sums,
                                                             _lib.compute_units(idx), ctypes.byref(out))
        need = out.value if st == _lib.OK else 0  # a shape the call itself refuses: let it say so
        if len(_BWD_NEED) >= 4096:
            _BWD_NEED.clear()
        _BWD_NEED[key] = need
    return need


def residual_norm_bwd(x_out: torch.Tensor, y: torch.Tensor, gh: torch.Tensor, gx: Optional[torch.Tensor] = None,
                      norm: str = "layer", post: Optional[str] = None, gate: Optional[torch.Tensor] = None,
                      scale: Optional[torch.Tensor] = None, w: Optional[torch.Tensor] = None,
                      b: Optional[torch.Tensor] = None, post_w: Optional[torch.Tensor] = None,
                      post_b: Optional[torch.Tensor] = None, alpha: float = 1.0, eps: float = 1e-6,
                      group_rows: int = 0, dx: Optional[torch.Tensor] = None,
                      dy: Optional[torch.Tensor] = None) -> ResidualNormGrads:
    """Gradients of residual_norm_fwd (regenvc_residual_norm_bwd), given those
    of h (gh, in y's type) and of x' from the rest of the program (gx, float32,
    or None).  x_out: the forward call's x'.  dx may be gx.  The gradients of
    the vectors are float32, [groups, C] (gate, scale, shift) and [C]; those of
    one kind share an allocation."""
    idx = _lib.index_of(x_out, "x_out")
    rows, C = x_out.shape
    act = y.dtype
    if act not in _ACT:
        raise ValueError(f"y must be bfloat16 or float32, got {act}")
    ldx, ldy = _lib.matrix(x_out, "x_out", torch.float32, rows, C, idx), _lib.matrix(y, "y", act, rows, C, idx)
    ldgh = _lib.matrix(gh, "gh", act, rows, C, idx)
    ldgx = 0 if gx is None else _lib.matrix(gx, "gx", torch.float32, rows, C, idx)
    dev = x_out.device
    if dx is None:
        dx, lddx = torch.empty(rows, C, dtype=torch.float32, device=dev), C
    else:
        lddx = _lib.matrix(dx, "dx", torch.float32, rows, C, idx)
    if dy is None:
        dy, lddy = torch.empty(rows, C, dtype=act, device=dev), C
    else:
        lddy = _lib.matrix(dy, "dy", act, rows, C, idx)
    groups, group_rows = _groups(rows, group_rows)
    v = _row_vectors(groups, C, group_rows, idx, gate, scale, None)
    np, nq = _norm(post, eps, post_w, post_b, C, "post", idx), _norm(norm, eps, w, b, C, "norm", idx)

    # what is asked for: of gate and modulation, of the weights
    make = torch.empty if rows > 0 else torch.zeros  # (sums over no rows)
    at = (gate is not None, scale is not None, scale is not None)
    at_rows = (w is not None, b is not None, post_w is not None, post_b is not None)
    ng, nr = sum(at), sum(at_rows)
    grouped = iter(make(ng, groups, C, dtype=torch.float32, device=dev).unbind(0)) if ng else None
    whole = iter(make(nr, C, dtype=torch.float32, device=dev).unbind(0)) if nr else None
    vec = [next(grouped) if on else None for on in at] + [next(whole) if on else None for on in at_rows]
    if rows > 0:
        grads = _lib.NormGrads(*[None if t is None else t.data_ptr() for t in vec])
        need = _bwd_need(rows, C, group_rows, ng, nr, idx)
        with _lib.on_device(idx):
            ws = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
            st = _lib.load().regenvc_residual_norm_bwd(
                x_out.data_ptr(), ldx, y.data_ptr(), ldy, _ACT[act], ctypes.byref(np), ctypes.byref(nq), ctypes.byref(v),
                alpha, gh.data_ptr(), ldgh, gx.data_ptr() if gx is not None else None, ldgx, dx.data_ptr(), lddx,
                dy.data_ptr(), lddy, ctypes.byref(grads), rows, C, ws.data_ptr() if ws is not None else None, need,
                _lib.raw_stream(idx))
        _lib.check(st, "regenvc_residual_norm_bwd")
    return ResidualNormGrads(dx, dy, *vec)


class DitBlock:
    """One diffusion-transformer block on the GPU: its bf16 parameters
    (device tensors, names as in regenvc_dit_params).  forward() runs
    regenvc_dit_block_fwd, updating the float32 residual stream in place, in
    a workspace of its own from torch's allocator on the current stream:
    calls from several streams or threads share no memory, and none is held
    between calls."""

    def __init__(self, params: Dict[str, torch.Tensor], heads: int = 12):
        missing = [n for n in _lib.DIT_PARAM_NAMES if n not in params]
        if missing:
            raise ValueError(f"missing parameters: {missing}")
        self.params = params
        self.C = params["w_o"].shape[0]
        self.F = params["w_1"].shape[0]
        self.heads = heads
        for n in _lib.DIT_PARAM_NAMES:
            t = params[n]
            if t.dtype != torch.bfloat16 or t.device.type != "cuda" or not t.is_contiguous():
                raise ValueError(f"parameter {n} must be a contiguous bf16 device tensor")
        self._c = _lib.DitParams(*[params[n].data_ptr() for n in _lib.DIT_PARAM_NAMES])
        self._ws = {}    # (device index, S, S_ctx) -> a workspace for such calls in place of their own
        self._need = {}  # (device index, S, S_ctx) -> workspace bytes

    def workspace_bytes(self, S: int, S_ctx: int, device, least: bool = False) -> int:
        """Workspace bytes of a forward pass (regenvc_dit_block_workspace), or
        the fewest that it takes (regenvc_dit_block_workspace_least)."""
        n_cu = torch.cuda.get_device_properties(device).multi_processor_count
        out = ctypes.c_int64()
        fn = "regenvc_dit_block_workspace_least" if least else "regenvc_dit_block_workspace"
        _lib.check(getattr(_lib.load(), fn)(S, S_ctx, self.C, self.heads, self.F, n_cu, ctypes.byref(out)), fn)
        return out.value

    def _workspace(self, S: int, S_ctx: int, device) -> torch.Tensor:
        key = (device.index, S, S_ctx)
        ws = self._ws.get(key)
        if ws is not None:
            return ws
        need = self._need.get(key)
        if need is None:
            need = self.workspace_bytes(S, S_ctx, device)
            if len(self._need) >= 4096:
                self._need.clear()
            self._need[key] = need
        try:
            return torch.empty(need, dtype=torch.uint8, device=device)
        except torch.OutOfMemoryError:  # without the linear layers' partial sums
            return torch.empty(self.workspace_bytes(S, S_ctx, device, least=True), dtype=torch.uint8, device=device)

    def forward(self, x: torch.Tensor, e: torch.Tensor, ctx_k: torch.Tensor, ctx_v: torch.Tensor, grid,
                token0: int = 0) -> torch.Tensor:
        """x: float32 [S, C] contiguous (updated in place); e: float32 [C];
        ctx_k, ctx_v: bf16 [S_ctx, heads, D] contiguous; grid = (frames,
        rows, cols) of the latent window."""
        S, C = x.shape
        S_ctx = ctx_k.shape[0]
        if C != self.C or x.dtype != torch.float32 or not x.is_contiguous():
            raise ValueError(f"x must be a contiguous float32 [S, {self.C}] tensor")
        for name, t in (("ctx_k", ctx_k), ("ctx_v", ctx_v)):
            if t.dtype != torch.bfloat16 or not t.is_contiguous() or t.numel() != S_ctx * C:
                raise ValueError(f"{name} must be a contiguous bf16 [S_ctx, heads, D] tensor")
        ws = self._workspace(S, S_ctx, x.device)
        gf, gh, gw = (int(v) for v in grid)
        st = _lib.load().regenvc_dit_block_fwd(
            x.data_ptr(), _vec(e, "e", torch.float32, C), ctypes.byref(self._c), ctx_k.data_ptr(), ctx_v.data_ptr(),
            S_ctx, S, C, self.heads, self.F, gf, gh, gw, int(token0), ws.data_ptr(), ws.numel(), _stream(x.device))
        _lib.check(st, "regenvc_dit_block_fwd")
        return x
