"""ctypes declarations of the C ABI in include/regenvc_attn.h."""
from __future__ import annotations

import ctypes
import os
import threading

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libregenvc_attn.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_HIP = 0, 1, 2, 3
BF16, F32 = 0, 1
MAX_PARTS = 16


class Tensor(ctypes.Structure):
    """regenvc_tensor: base pointer + element strides of the b, s, h axes."""
    _fields_ = [("ptr", ctypes.c_void_p), ("stride_b", ctypes.c_int64),
                ("stride_s", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class AttnPlan(ctypes.Structure):
    """regenvc_attn_plan: the work decomposition of one attention call."""
    _fields_ = [("query_tiles", ctypes.c_int32), ("key_tiles", ctypes.c_int32),
                ("whole_tiles", ctypes.c_int32), ("split_tiles", ctypes.c_int32),
                ("key_ranges", ctypes.c_int32), ("workspace_bytes", ctypes.c_int64),
                ("tile_rows", ctypes.c_int32)]


class TilePlan(ctypes.Structure):
    """regenvc_tile_plan: the decomposition of a matrix product."""
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "cols", "waves", "k_ranges")]


class VaeTile(ctypes.Structure):
    """regenvc_vae_tile: a tile's core and region (half-open row/column ranges)."""
    _fields_ = [(n, ctypes.c_int32) for n in ("core_y0", "core_y1", "core_x0", "core_x1",
                                              "reg_y0", "reg_y1", "reg_x0", "reg_x1")]


DIT_PARAM_NAMES = ("w_mod", "b_mod", "w_qkv", "b_qkv", "w_qn", "w_kn", "w_o", "b_o", "w_n3", "b_n3", "w_qc",
                   "b_qc", "w_qcn", "w_oc", "b_oc", "w_1", "b_1", "w_2", "b_2")


class DitParams(ctypes.Structure):
    """regenvc_dit_params: device pointers of one block's bf16 parameters."""
    _fields_ = [(n, ctypes.c_void_p) for n in DIT_PARAM_NAMES]


class MxCache(ctypes.Structure):
    """regenvc_mx_cache: device pointers and sizes of an MXFP4 key/value cache."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_codes", "k_scales", "v_codes", "v_scales")] + \
               [(n, ctypes.c_int32) for n in ("B", "capacity", "heads", "D")]


class MxAttnPlan(ctypes.Structure):
    """regenvc_mx_attn_plan: the decomposition of an attention call over a cache."""
    _fields_ = [(n, ctypes.c_int32) for n in ("tile_rows", "row_tiles", "key_ranges")]


class PagePool(ctypes.Structure):
    """regenvc_page_pool: device pointers and sizes of a bf16 key/value cache in pages."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "means")] + \
               [(n, ctypes.c_int32) for n in ("pages", "page", "heads", "D")]


class PageBatch(ctypes.Structure):
    """regenvc_page_batch: the sequences of a call."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("table", "first", "lens")] + [("table_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("B", "columns", "T")]


class RotaryTable(ctypes.Structure):
    """regenvc_rotary: turns per position of the rotated pairs of a head."""
    _fields_ = [("turns", ctypes.c_void_p), ("pairs", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("amplitude", ctypes.c_float)]


class PagedAttnShape(ctypes.Structure):
    """regenvc_paged_attn_shape: what the plan of an attention call over pages goes by."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "H", "heads", "D", "page", "q_block", "count", "max_rows",
                                              "max_len", "causal")]


class PagedAttnPlan(ctypes.Structure):
    """regenvc_paged_attn_plan: the decomposition of attention over pages."""
    _fields_ = [(n, ctypes.c_int32) for n in ("tile_rows", "workgroups", "split")]


class Norm(ctypes.Structure):
    """regenvc_norm: a norm over a row, with its bf16 weights."""
    _fields_ = [("kind", ctypes.c_int32), ("eps", ctypes.c_float), ("w", ctypes.c_void_p), ("b", ctypes.c_void_p)]


class RowVectors(ctypes.Structure):
    """regenvc_row_vectors: gate and modulation of the rows, one set per group."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("gate", "scale", "shift")] + \
               [("ld", ctypes.c_int64), ("group_rows", ctypes.c_int32)]


NORM_GRAD_NAMES = ("dgate", "dscale", "dshift", "dw", "db", "dpost_w", "dpost_b")


class NormGrads(ctypes.Structure):
    """regenvc_norm_grads: f32 gradients of a norm's vectors."""
    _fields_ = [(n, ctypes.c_void_p) for n in NORM_GRAD_NAMES]


class RegenvcError(RuntimeError):
    def __init__(self, status: int, fn: str, detail: str):
        self.status = status
        super().__init__(f"{fn} failed with status {status}: {detail}")


_PT = ctypes.POINTER(Tensor)
_i32 = ctypes.c_int32
_FP = ctypes.POINTER(ctypes.c_float)
_p = ctypes.c_void_p
_i64 = ctypes.c_int64
_PI64 = ctypes.POINTER(ctypes.c_int64)
_PC = ctypes.POINTER(MxCache)
_PN = ctypes.POINTER(Norm)
_PP, _PB, _PR = ctypes.POINTER(PagePool), ctypes.POINTER(PageBatch), ctypes.POINTER(RotaryTable)
_PS = ctypes.POINTER(PagedAttnShape)
_SIGNATURES = {
    "regenvc_attn_fwd": [_PT, _PT, _PT, _PT, ctypes.c_int, ctypes.c_void_p,
                         _i32, _i32, _i32, _i32, _i32, ctypes.c_float, ctypes.c_void_p],
    "regenvc_attn_fwd_noalloc": [_PT, _PT, _PT, _PT, ctypes.c_int, ctypes.c_void_p,
                                 _i32, _i32, _i32, _i32, _i32, ctypes.c_float, ctypes.c_void_p],
    "regenvc_attn_partial_fwd": [_PT, _PT, _PT, _PT, ctypes.c_void_p,
                                 _i32, _i32, _i32, _i32, _i32, ctypes.c_float, ctypes.c_void_p],
    "regenvc_attn_partials_fwd": [_PT, _PT, _PT, _i32, ctypes.POINTER(_i32), ctypes.POINTER(ctypes.c_void_p),
                                  ctypes.POINTER(ctypes.c_void_p), _i32, _i32, _i32, _i32, _i32, ctypes.c_float,
                                  ctypes.c_void_p],
    "regenvc_attn_partials_plan_query": [_i32, _i32, _i32, _i32, ctypes.POINTER(_i32), _i32, _i32,
                                         ctypes.POINTER(AttnPlan)],
    "regenvc_lse_merge": [ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_void_p), _i32,
                          _PT, ctypes.c_int, ctypes.c_void_p, _i32, _i32, _i32, _i32, ctypes.c_void_p],
    "regenvc_attn_ring_accumulate": [_PT, _PT, _PT, _PT, ctypes.c_void_p, _PT, ctypes.c_int,
                                     _i32, _i32, _i32, _i32, _i32, ctypes.c_float, ctypes.c_void_p],
    "regenvc_cross_attn_dual_fwd": [_PT, _PT, _PT, _i32, _PT, _PT, _i32, _PT, ctypes.c_void_p, ctypes.c_void_p,
                                    _i32, _i32, _i32, _i32, ctypes.c_float, ctypes.c_void_p],
    "regenvc_cross_attn_fwd": [_PT, _PT, _PT, _PT, ctypes.c_int, ctypes.c_void_p,
                               _i32, _i32, _i32, _i32, _i32, ctypes.c_float, ctypes.c_void_p],
    "regenvc_attn_plan_query": [_i32, _i32, _i32, _i32, _i32, _i32, ctypes.POINTER(AttnPlan)],
    "regenvc_cross_attn_dual_plan_query": [_i32, _i32, _i32, _i32, _i32, _i32, _i32, ctypes.POINTER(AttnPlan)],
    "regenvc_attn_set_workspace": [ctypes.c_void_p, ctypes.c_int64],
    "regenvc_linear_fwd": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                           ctypes.c_void_p, ctypes.c_int64, _i32, _i32, _i32, _i32, ctypes.c_void_p],
    "regenvc_linear_fwd_ws": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                              ctypes.c_void_p, ctypes.c_int64, _i32, _i32, _i32, _i32, ctypes.c_void_p,
                              ctypes.c_int64, ctypes.c_void_p],
    "regenvc_linear_workspace": [_i32, _i32, _i32, _i32, _i32, ctypes.POINTER(ctypes.c_int64)],
    "regenvc_linear_plan_query": [_i32, _i32, _i32, _i32, _i32, ctypes.c_int64, ctypes.POINTER(TilePlan)],
    "regenvc_layer_norm_fwd": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                               ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, _i32, _i32, ctypes.c_float,
                               ctypes.c_void_p],
    "regenvc_rms_norm_fwd": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                             _i32, _i32, ctypes.c_float, ctypes.c_void_p],
    "regenvc_dit_modulation": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, _i32, _i32,
                               ctypes.c_void_p],
    "regenvc_vae_split": [_i32, _i32, _i32, _i32, _i32, ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32),
                          ctypes.POINTER(ctypes.c_int32)],
    "regenvc_vae_conv3d_fwd": [ctypes.c_void_p, _i32, ctypes.c_void_p, ctypes.c_void_p, _i32, ctypes.c_void_p,
                               _i32, _i32, _i32, _i32, _i32, ctypes.c_void_p, _i32, _i32, _i32, ctypes.c_void_p,
                               ctypes.c_int64, ctypes.c_void_p],
    "regenvc_vae_conv3d_workspace": [_i32, _i32, _i32, _i32, _i32, _i32, _i32, ctypes.POINTER(ctypes.c_int64)],
    "regenvc_vae_conv3d_plan_query": [_i32, _i32, _i32, _i32, _i32, _i32, _i32, ctypes.c_int64,
                                      ctypes.POINTER(TilePlan)],
    "regenvc_vae_blend": [ctypes.c_void_p, ctypes.c_void_p, _i32, _i32, _i32, _i32, _i32, _i32, _i32, _i32,
                          ctypes.c_void_p, ctypes.c_void_p],
    "regenvc_dit_block_workspace": [_i32, _i32, _i32, _i32, _i32, _i32, ctypes.POINTER(ctypes.c_int64)],
    "regenvc_dit_block_workspace_least": [_i32, _i32, _i32, _i32, _i32, _i32, ctypes.POINTER(ctypes.c_int64)],
    "regenvc_dit_block_fwd": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                              _i32, _i32, _i32, _i32, _i32, _i32, _i32, _i32, _i32, ctypes.c_void_p,
                              ctypes.c_int64, ctypes.c_void_p],
    "regenvc_qk_norm_rope": [_PT, _PT, ctypes.c_void_p, ctypes.c_void_p, _PT, _PT, _i32, _i32, _i32, _i32,
                             _i32, _i32, _i32, _i32, ctypes.c_float, ctypes.c_float, ctypes.c_void_p],
    "regenvc_residual_norm_fwd": [_p, _i64, _p, _i64, ctypes.c_int, _PN, _PN, ctypes.POINTER(RowVectors), ctypes.c_float,
                                  _p, _i64, _p, _i64, _i32, _i32, _p],
    "regenvc_residual_norm_bwd": [_p, _i64, _p, _i64, ctypes.c_int, _PN, _PN, ctypes.POINTER(RowVectors), ctypes.c_float,
                                  _p, _i64, _p, _i64, _p, _i64, _p, _i64, ctypes.POINTER(NormGrads), _i32, _i32, _p,
                                  _i64, _p],
    "regenvc_residual_norm_bwd_workspace": [_i32, _i32, _i32, _i32, _i32, _i32, _PI64],
    "regenvc_mx_bytes": [_i32, _i32, _PI64, _PI64],
    "regenvc_mx_quantize": [_p, ctypes.c_int, _i64, _p, _p, _i32, _i32, _p],
    "regenvc_mx_dequantize": [_p, _p, _p, ctypes.c_int, _i64, _i32, _i32, _p],
    "regenvc_mx_linear_fwd": [_p, _i64, _p, _p, _p, _p, _p, _p, _p, _i64, _i32, _i32, _i32, _i32, _p, _i64, _p],
    "regenvc_mx_linear_workspace": [_i32, _i32, _i32, _i32, _PI64],
    "regenvc_mx_linear_plan_query": [_i32, _i32, _i32, _i32, _i32, ctypes.POINTER(TilePlan)],
    "regenvc_mx_cache_append": [_PC, _PT, _PT, _i32, _p, _p, _p],
    "regenvc_mx_cache_values": [_PC, _p, _p, ctypes.c_int, _p],
    "regenvc_mx_attn_cache_fwd": [_PT, _PC, _p, _i32, _PT, ctypes.c_int, _p, _i32, _i32, _i32, ctypes.c_float, _p, _i64,
                                  _p],
    "regenvc_mx_attn_cache_workspace": [_i32, _i32, _i32, _i32, _i32, _i32, _i32, _PI64],
    "regenvc_mx_attn_cache_plan_query": [_i32, _i32, _i32, _i32, _i32, _i32, _i32, ctypes.POINTER(MxAttnPlan)],
    "regenvc_paged_append": [_PP, _PB, _PT, _PT, _PT, _p, _p, ctypes.c_float, _PR, _PT, _i32, _p],
    "regenvc_paged_select": [_PT, _PP, _PB, _i32, _i32, _i32, _i32, _i32, _i32, _p, _p],
    "regenvc_paged_attn_fwd": [_PT, _PP, _PB, _p, _i32, _i32, _i32, _i32, _i32, _PT, ctypes.c_int, _p, _i32,
                               ctypes.c_float, _p, _i64, _p],
    "regenvc_paged_attn_workspace": [_PS, _i32, _PI64],
    "regenvc_paged_attn_plan_query": [_PS, _i32, ctypes.POINTER(PagedAttnPlan)],
}

_lib = None


def load(path: str | None = None) -> ctypes.CDLL:
    """Loads the built library (once).  Fails loudly if it has not been built:
    there is no fallback implementation."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise ImportError(f"{p} is missing; build it with `python -m paper_2607_28144_amd.build`")
    lib = ctypes.CDLL(p)
    for name, argtypes in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.argtypes = argtypes
        fn.restype = ctypes.c_int
    lib.regenvc_status_str.argtypes = [ctypes.c_int]
    lib.regenvc_status_str.restype = ctypes.c_char_p
    lib.regenvc_last_error.argtypes = []
    lib.regenvc_last_error.restype = ctypes.c_char_p
    lib.regenvc_attn_pool_draws.argtypes = []
    lib.regenvc_attn_pool_draws.restype = ctypes.c_int64
    if path is None:
        _lib = lib
    return lib


def stream_of(device) -> int:
    """torch's current stream of a device, as the address the C ABI takes.
    (The raw query where this torch has it: building a Stream object per call
    costs more than the launch.)"""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is not None and device.index is not None:
        return raw(device.index)
    return torch.cuda.current_stream(device).cuda_stream


class _Nothing:
    def __enter__(self):
        return self

    def __exit__(self, *exc):
        return False


_NOTHING = _Nothing()
_current_device = None


def on_device(device):
    """Context with a torch device (or the device of an index) current; nothing to do where it is already."""
    global _current_device
    if _current_device is None:
        import torch
        torch.cuda.current_device()  # initializes
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    if _current_device() == (device if type(device) is int else device.index):
        return _NOTHING
    import torch
    return torch.cuda.device(device)


def index_of(t, name: str) -> int:
    """The index of the device that a tensor lies on."""
    idx = t.get_device()
    if idx < 0:
        raise ValueError(f"{name} must be a device tensor, got {t.device}")
    return idx


def int32(**sizes: int) -> None:
    """Refuses sizes that do not fit the int32 arguments of the C ABI: ctypes would hand on their low 32 bits."""
    for name, v in sizes.items():
        if not -(1 << 31) <= v < 1 << 31:
            raise ValueError(f"{name}={v} does not fit 32 bits")


def matrix(t, name: str, dtype, rows: int, cols: int, idx: int) -> int:
    """The row stride of a [rows, cols] tensor of this type on device idx; refuses any other.  (Of a single row, whose
    stride torch leaves to chance: cols.)"""
    s, st = t.shape, t.stride()
    if t.dtype is dtype and t.get_device() == idx and len(st) == 2 and s[0] == rows and s[1] == cols \
            and (st[1] == 1 or cols <= 1):
        return st[0] if rows > 1 else cols
    raise ValueError(f"{name} must be a {dtype} tensor [{rows}, {cols}] with unit column stride on cuda:{idx}, got "
                     f"{t.dtype} {tuple(s)} on {t.device}")


def vector(t, name: str, dtype, n: int, idx: int):
    """The address of a contiguous tensor of n elements of this type on device idx (None for None); refuses any other."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == idx and t.numel() == n and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements on cuda:{idx}, got {t.dtype} "
                     f"{tuple(t.shape)} on {t.device}")


_N_CU = {}  # device index -> compute units


def compute_units(idx: int) -> int:
    """Compute units of the device of an index."""
    n = _N_CU.get(idx)
    if n is None:
        import torch
        n = _N_CU[idx] = torch.cuda.get_device_properties(idx).multi_processor_count
    return n


_raw_stream = None


def raw_stream(idx: int) -> int:
    """torch's current stream of the device of an index, as the address the C ABI takes."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda i: torch.cuda.current_stream(i).cuda_stream)
    return _raw_stream(idx)


def split_workspace(need: int, device):
    """`need` bytes for the partial sums of a call that can also run without
    splitting K, from torch's allocator on the current stream; None where
    none are needed or the device has no room for them."""
    import torch
    if need <= 0:
        return None
    try:
        return torch.empty(need, dtype=torch.uint8, device=device)
    except torch.OutOfMemoryError:
        return None


_kept = threading.local()


def keep_error_detail() -> None:
    """Saves the library's error text of the failed call just made on this
    thread, for the next check() (a later successful call clears the text)."""
    _kept.detail = load().regenvc_last_error().decode(errors="replace")


def check(status: int, fn: str) -> None:
    kept = getattr(_kept, "detail", None)
    _kept.detail = None
    if status != OK:
        detail = kept if kept is not None else load().regenvc_last_error().decode(errors="replace")
        raise RegenvcError(status, fn, detail)
