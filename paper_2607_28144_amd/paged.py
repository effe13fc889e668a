"""Thin torch-facing binding of the kernels of a bf16 key/value cache in pages
(include/regenvc_paged.h): argument marshalling only; every step runs in the
HIP kernels of libregenvc_attn.so on torch's current stream.

A pool (PagedCache) holds pages; the caller keeps which pages a sequence has, as
three int32 device tensors that all calls take:
  table [B, columns]  row b: the pages of sequence b in order
  first [B + 1]       the new tokens of sequence b are rows first[b] ..
                      first[b + 1] - 1 of the packed [T, heads, D] tensors
  lens [B]            its places, the new tokens' (the last ones) among them
Rows of no sequence are left as they are in outputs that the caller gives.
Workspaces are torch allocations on the current stream.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple

import torch

from . import _lib
from .api import _DT, _scale


class PagedCache:
    """Keys and values of `pages` pages of `page` places for `heads` key heads
    (regenvc_page_pool): k, v bf16 [pages, heads, page, D], contiguous device
    tensors; means bf16 [pages, heads, D], or None where no pages are selected."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, means: Optional[torch.Tensor] = None):
        if k.dim() != 4 or v.shape != k.shape:
            raise ValueError(f"k, v must be [pages, heads, page, D], got {tuple(k.shape)}, {tuple(v.shape)}")
        self.pages, self.heads, self.page, self.D = k.shape
        idx = _lib.index_of(k, "k")
        _lib.vector(k, "k", torch.bfloat16, k.numel(), idx)
        _lib.vector(v, "v", torch.bfloat16, k.numel(), idx)
        if means is not None:
            if tuple(means.shape) != (self.pages, self.heads, self.D):
                raise ValueError(f"means must be {(self.pages, self.heads, self.D)}, got {tuple(means.shape)}")
            _lib.vector(means, "means", torch.bfloat16, means.numel(), idx)
        _lib.int32(pages=self.pages, heads=self.heads, page=self.page, D=self.D)
        self.device = k.device
        self._parts = k, v, means
        self._c = _lib.PagePool(k.data_ptr(), v.data_ptr(), None if means is None else means.data_ptr(), self.pages, self.page,
                                self.heads, self.D)

    @classmethod
    def zeros(cls, pages: int, page: int, heads: int, D: int, means: bool = False, device="cuda") -> "PagedCache":
        """A pool of zeros."""
        k, v = (torch.zeros(pages, heads, page, D, dtype=torch.bfloat16, device=device) for _ in range(2))
        return cls(k, v, torch.zeros(pages, heads, D, dtype=torch.bfloat16, device=device) if means else None)

    # read-only: the addresses of the tensors are in what the calls get
    k = property(lambda self: self._parts[0])
    v = property(lambda self: self._parts[1])
    means = property(lambda self: self._parts[2])


class Rotary:
    """Rotation of the first `dim` channels of a head (regenvc_rotary): pair i
    of the token at place p by the angle p f_i, f_i = theta^(-2 i / dim).

      layout   "interleaved": pair i is channels 2 i and 2 i + 1; "half": i and
               dim / 2 + i
      scaling  for contexts `factor` times those of training (of original_len
               tokens, "parts" only):
               "linear" f_i / factor
               "base"   theta factor^(dim / (dim - 2)) in theta's place
               "parts"  f_i where a pair turns `fast` times or more within
                        original_len, f_i / factor where it does so `slow` times or
                        less, mixed linearly by that number of turns (not by the
                        pair's index) between; the rotated channels of queries and
                        keys times 1 + ln(factor) / 10
    """

    def __init__(self, dim: int, theta: float = 10000.0, layout: str = "half", scaling: Optional[str] = None,
                 factor: float = 1.0, original_len: Optional[int] = None, fast: float = 32.0, slow: float = 1.0,
                 device="cuda"):
        if layout not in ("half", "interleaved"):
            raise ValueError(f"layout {layout!r} (half or interleaved)")
        if scaling not in (None, "linear", "base", "parts"):
            raise ValueError(f"scaling {scaling!r} (None, linear, base or parts)")
        if dim < 0 or dim % 16 != 0:
            raise ValueError(f"dim={dim} is not a multiple of 16")
        if not (theta > 0 and factor > 0):
            raise ValueError(f"theta={theta} and factor={factor} must be positive")
        if scaling is None and factor != 1.0:
            raise ValueError(f"factor={factor} needs a scaling")
        if scaling == "parts" and (original_len is None or original_len < 1 or not fast > slow or factor < 1):
            raise ValueError("parts needs original_len, fast > slow and factor >= 1")
        self.dim, self.layout, self.amplitude = int(dim), layout, 1.0
        base = theta * factor ** (dim / (dim - 2)) if scaling == "base" else theta
        turns = base ** (-2 * torch.arange(dim // 2, dtype=torch.float64) / max(dim, 1)) / (2 * math.pi)
        if scaling == "linear":
            turns = turns / factor
        elif scaling == "parts":
            keep = torch.clamp((turns * original_len - slow) / (fast - slow), 0.0, 1.0)
            turns = turns * (keep + (1.0 - keep) / factor)
            self.amplitude = 1.0 + 0.1 * math.log(factor)
        self.turns = turns.to(device)  # double: whole turns of far places are taken off in 64 bits
        self._c = _lib.RotaryTable(self.turns.data_ptr(), self.dim // 2, int(layout == "interleaved"), self.amplitude)


_BF16, _INT32 = torch.bfloat16, torch.int32


def _packed(t: torch.Tensor, name: str, shape: Tuple[int, int, int], idx: int, dtype=_BF16) -> _lib.Tensor:
    """The descriptor of a [T, heads, D] tensor of this type on device idx; refuses any other."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == idx:
        st = t.stride()
        if st[2] == 1:  # of a single row or head, whose stride torch leaves to chance: any
            return _lib.Tensor(t.data_ptr(), 0, st[0] if shape[0] > 1 else 0, st[1] if shape[1] > 1 else 0)
    raise ValueError(f"{name} must be a {dtype} tensor {list(shape)} with unit channel stride on cuda:{idx}, got {t.dtype} "
                     f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _batch(table, first, lens, T: int, idx: int) -> _lib.PageBatch:
    """The descriptor of a call's sequences on device idx; refuses any other tensors."""
    s = table.shape
    if len(s) != 2:
        raise ValueError(f"table must be [B, columns], got {tuple(s)}")
    B, columns = s
    if B >= 1 << 31 or columns >= 1 << 31 or T >= 1 << 31:
        _lib.int32(B=B, columns=columns, T=T)
    stride = _lib.matrix(table, "table", _INT32, B, columns, idx)
    return _lib.PageBatch(table.data_ptr(), _lib.vector(first, "first", _INT32, B + 1, idx),
                          _lib.vector(lens, "lens", _INT32, B, idx), stride, B, columns, T)


def _index(cache: PagedCache) -> int:
    return cache.device.index


def append(cache: PagedCache, table: torch.Tensor, first: torch.Tensor, lens: torch.Tensor, k: torch.Tensor,
           v: torch.Tensor, q: Optional[torch.Tensor] = None, w_q: Optional[torch.Tensor] = None,
           w_k: Optional[torch.Tensor] = None, eps: float = 1e-6, rotary: Optional[Rotary] = None,
           q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """New tokens to the cache in one pass (regenvc_paged_append): each head of
    q and k (bf16 [T, heads, D], views of a fused projection as well) normed with
    the weights w_q, w_k (bf16 [D]; None: not normed) and rotated at its token's
    place, k and v to their places, the mean keys of the touched pages taken anew
    where the cache has means.  Returns q's (q_out, which may be q; a new tensor if
    None; None without q)."""
    idx = _index(cache)
    D = cache.D
    T = k.shape[0]
    n = _batch(table, first, lens, T, idx)
    kd = _packed(k, "k", (T, cache.heads, D), idx)
    vd = _packed(v, "v", (T, cache.heads, D), idx)
    H, qd, od = 0, None, None
    if q is not None:
        H = q.shape[1] if q.dim() == 3 else 0
        qd = ctypes.byref(_packed(q, "q", (T, H, D), idx))
        if q_out is None:
            q_out = torch.empty(T, H, D, dtype=_BF16, device=cache.device)
            od = ctypes.byref(_lib.Tensor(q_out.data_ptr(), 0, H * D, D))
        else:
            od = ctypes.byref(_packed(q_out, "q_out", (T, H, D), idx))
        if H == 0:
            qd = od = None
    elif q_out is not None:
        raise ValueError("q_out without q")
    wq = _lib.vector(w_q, "w_q", _BF16, D, idx)
    wk = _lib.vector(w_k, "w_k", _BF16, D, idx)
    rc = None
    if rotary is not None:
        if rotary.turns.get_device() != idx:
            raise ValueError(f"the rotary table is on {rotary.turns.device}, the cache on {cache.device}")
        rc = ctypes.byref(rotary._c)
    with _lib.on_device(idx):
        st = _lib.load().regenvc_paged_append(
            ctypes.byref(cache._c), ctypes.byref(n), qd, ctypes.byref(kd), ctypes.byref(vd), wq, wk, eps, rc, od, H,
            _lib.raw_stream(idx))
    _lib.check(st, "regenvc_paged_append")
    return q_out


_NEED = {}  # (device index, shape) -> workspace bytes of a call


def _need(shape: tuple, idx: int) -> int:
    key = (idx, shape)
    need = _NEED.get(key)
    if need is None:
        out = ctypes.c_int64()
        st = _lib.load().regenvc_paged_attn_workspace(ctypes.byref(_lib.PagedAttnShape(*shape)), _lib.compute_units(idx),
                                                      ctypes.byref(out))
        need = out.value if st == _lib.OK else 0  # a shape the call itself refuses: let it say so
        if len(_NEED) >= 4096:
            _NEED.clear()
        _NEED[key] = need
    return need


def _attn(q, cache, table, first, lens, chosen, q_block, causal, scale, max_rows, max_len, out_dtype, out, return_lse,
          lse_out):
    idx = _index(cache)
    if q.dim() != 3:
        raise ValueError(f"q must be [T, H, D], got {tuple(q.shape)}")
    T, H, D = q.shape
    n = _batch(table, first, lens, T, idx)
    qd = _packed(q, "q", (T, H, cache.D), idx)
    if out_dtype not in _DT:
        raise TypeError(f"out_dtype must be bfloat16 or float32, got {out_dtype}")
    if out is None:
        out = torch.empty(T, H, D, dtype=out_dtype, device=cache.device)
        od = _lib.Tensor(out.data_ptr(), 0, H * D, D)
    else:
        od = _packed(out, "out", (T, H, D), idx, out_dtype)
    if lse_out is not None:
        if tuple(lse_out.shape) != (H, T):
            raise ValueError(f"lse must be {(H, T)}, got {tuple(lse_out.shape)}")
        lp = _lib.vector(lse_out, "lse", torch.float32, H * T, idx)
    elif return_lse:
        lse_out = torch.empty(H, T, dtype=torch.float32, device=cache.device)
        lp = lse_out.data_ptr()
    else:
        lp = None
    count, sp = 0, None
    if chosen is not None:
        count = chosen.shape[2] if chosen.dim() == 3 else 0
        _lib.int32(q_block=q_block, count=count)
        # (a list without entries has no address, which the call reads as every page)
        if q_block < 1 or count < 1 or tuple(chosen.shape) != (T // q_block + n.B, cache.heads, count):
            raise ValueError(f"selected must be [T // q_block + B, heads, count], got {tuple(chosen.shape)} for q_block={q_block}")
        sp = _lib.vector(chosen, "selected", torch.int32, chosen.numel(), idx)
    rows = T if max_rows is None else int(max_rows)
    places = n.columns * cache.page if max_len is None else int(max_len)
    if H >= 1 << 31 or not 0 <= rows < 1 << 31 or not 0 <= places < 1 << 31:
        _lib.int32(H=H, max_rows=rows, max_len=places)
    need = _need((n.B, T, H, cache.heads, D, cache.page, q_block, count, rows, places, int(causal)), idx)
    with _lib.on_device(idx):
        ws = torch.empty(need, dtype=torch.uint8, device=cache.device) if need > 0 else None
        st = _lib.load().regenvc_paged_attn_fwd(
            ctypes.byref(qd), ctypes.byref(cache._c), ctypes.byref(n), sp, q_block, count, int(causal), rows, places,
            ctypes.byref(od), _DT[out_dtype], lp, H, _scale(scale, D), ws.data_ptr() if ws is not None else None, need,
            _lib.raw_stream(idx))
    _lib.check(st, "regenvc_paged_attn_fwd")
    return out, lse_out


def attn_fwd(q: torch.Tensor, cache: PagedCache, table: torch.Tensor, first: torch.Tensor, lens: torch.Tensor,
             causal: bool = True, scale: Optional[float] = None, max_rows: Optional[int] = None,
             max_len: Optional[int] = None, out_dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
             return_lse: bool = True, lse_out: Optional[torch.Tensor] = None
             ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Attention of q (bf16 [T, H, D]; H a multiple of the cache's heads) to the
    places of its sequence, up to each token's own or, with causal=False, all of
    them (regenvc_paged_attn_fwd).  max_rows and max_len (default: T and the
    table's places) are the most new tokens and places of a sequence that the work
    is planned for.  Returns O [T, H, D] and LSE [H, T] (or None); a query that
    sees no place gives 0 and -inf."""
    return _attn(q, cache, table, first, lens, None, 1, causal, scale, max_rows, max_len, out_dtype, out, return_lse, lse_out)


def select_pages(q: torch.Tensor, cache: PagedCache, table: torch.Tensor, first: torch.Tensor, lens: torch.Tensor,
                 count: int, q_block: int = 1, keep_first: int = 1, keep_last: int = 1, causal: bool = True,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The pages that each block of q_block queries of a sequence reads, for
    every key head: the first keep_first and the last keep_last that it sees, and
    of the others those whose mean key has the largest product with the block's
    queries, `count` in all (regenvc_paged_select).  int32 [T // q_block + B, heads,
    count], ascending, -1 behind the last; block i of sequence b is first[b] //
    q_block + b + i.  The last pages are counted from a block's last query: for each
    query of a causal call to keep the page that it stands in, keep_last has to be
    ceil((q_block - 1) / page) + 1, more than the default of 1 where q_block is."""
    idx = _index(cache)
    if q.dim() != 3:
        raise ValueError(f"q must be [T, H, D], got {tuple(q.shape)}")
    T, H, _ = q.shape
    n = _batch(table, first, lens, T, idx)
    qd = _packed(q, "q", (T, H, cache.D), idx)
    _lib.int32(H=H, count=count, q_block=q_block, keep_first=keep_first, keep_last=keep_last)
    if q_block < 1 or count < 0:
        raise ValueError(f"q_block={q_block}, count={count}")
    if cache.means is None:
        raise ValueError("the cache has no means")
    shape = (T // q_block + n.B, cache.heads, count)
    if out is None:
        out = torch.empty(shape, dtype=torch.int32, device=cache.device)
    elif tuple(out.shape) != shape:
        raise ValueError(f"out must be {shape}, got {tuple(out.shape)}")
    op = _lib.vector(out, "out", torch.int32, out.numel(), idx)
    with _lib.on_device(idx):
        st = _lib.load().regenvc_paged_select(ctypes.byref(qd), ctypes.byref(cache._c), ctypes.byref(n), H, q_block, count,
                                              keep_first, keep_last, int(causal), op, _lib.raw_stream(idx))
    _lib.check(st, "regenvc_paged_select")
    return out


def attn_pages_fwd(q: torch.Tensor, cache: PagedCache, table: torch.Tensor, first: torch.Tensor, lens: torch.Tensor,
                   selected: torch.Tensor, q_block: int = 1, causal: bool = True, scale: Optional[float] = None,
                   max_rows: Optional[int] = None, max_len: Optional[int] = None,
                   out_dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None, return_lse: bool = True,
                   lse_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """attn_fwd in which the queries of a block see only the pages that
    `selected` (int32 [T // q_block + B, heads, count], as from select_pages)
    names for it and their key head: indices into the sequence's row of the table,
    -1 for none (regenvc_paged_attn_fwd)."""
    if selected is None:
        raise ValueError("selected is None (attn_fwd attends to every page)")
    return _attn(q, cache, table, first, lens, selected, q_block, causal, scale, max_rows, max_len, out_dtype, out, return_lse,
                 lse_out)
