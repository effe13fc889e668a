"""Host side of include/regenvc_mx.h and of the residual-norm entry points on
the CPU: every declared symbol is there, bad arguments are refused before any
HIP call (the fake addresses are never dereferenced), and the plans are sound."""
import ctypes
import os
import re

import pytest

from conftest import REPO
from paper_2607_28144_amd import _lib

F = 0x10000000    # 256-byte aligned, never dereferenced
G = F + (1 << 32)
H = F + (1 << 33)
I = F + (1 << 34)
BIG = 1 << 62


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def refused(lib, status, word, st):
    assert st == status, (st, lib.regenvc_last_error())
    assert word in lib.regenvc_last_error().decode(), lib.regenvc_last_error()


INV, UNS = _lib.ERR_INVALID_ARG, _lib.ERR_UNSUPPORTED


def test_every_declared_symbol_is_bound(lib):
    text = "".join(open(os.path.join(REPO, "include", h)).read() for h in ("regenvc_mx.h", "regenvc_dit.h"))
    names = set(re.findall(r"^regenvc_status\s+(regenvc_\w+)\s*\(", text, re.M))
    assert {"regenvc_mx_linear_fwd", "regenvc_mx_attn_cache_fwd", "regenvc_residual_norm_bwd"} <= names
    for n in names:
        assert hasattr(lib, n) and n in _lib._SIGNATURES


def test_mx_bytes(lib):
    c, s = ctypes.c_int64(), ctypes.c_int64()
    for rows, K, nc, ns in [(0, 64, 0, 0), (1, 8, 128, 128), (17, 256, 17 * 128, 256), (100, 264, 100 * 256, 7 * 256),
                            (5, 0, 0, 0), (16, 8960, 16 * 4480, 35 * 128)]:
        assert lib.regenvc_mx_bytes(rows, K, ctypes.byref(c), ctypes.byref(s)) == 0 and (c.value, s.value) == (nc, ns)
    refused(lib, INV, "NULL", lib.regenvc_mx_bytes(1, 8, None, ctypes.byref(s)))
    refused(lib, INV, "negative", lib.regenvc_mx_bytes(-1, 8, ctypes.byref(c), ctypes.byref(s)))
    refused(lib, UNS, "multiple of 8", lib.regenvc_mx_bytes(1, 12, ctypes.byref(c), ctypes.byref(s)))
    refused(lib, UNS, "multiple of 8", lib.regenvc_mx_bytes(1, (1 << 20) + 8, ctypes.byref(c), ctypes.byref(s)))


def test_quantize_refusals(lib):
    q = lib.regenvc_mx_quantize
    ok = dict(x=F, t=0, ld=64, c=G, s=H, rows=4, K=64)

    def call(**kw):
        a = dict(ok, **kw)
        return q(a["x"], a["t"], a["ld"], a["c"], a["s"], a["rows"], a["K"], None)
    refused(lib, INV, "dtype", call(t=7))
    refused(lib, INV, "negative", call(rows=-1))
    refused(lib, UNS, "ldx", call(ld=60))
    refused(lib, UNS, "ldx", call(ld=56))
    refused(lib, INV, "NULL", call(c=None))
    refused(lib, UNS, "aligned", call(x=F + 8))
    refused(lib, UNS, "aligned", call(s=H + 1))
    refused(lib, INV, "overlap", call(c=F))
    refused(lib, INV, "overlap", call(s=F + 64))
    assert call(rows=0) == 0 and call(K=0, ld=1) == 0
    d = lib.regenvc_mx_dequantize
    refused(lib, INV, "overlap", d(F, G, F + 16, 1, 64, 4, 64, None))
    refused(lib, UNS, "ldo", d(F, G, H, 1, 32, 4, 64, None))
    refused(lib, INV, "NULL", d(F, None, H, 1, 64, 4, 64, None))


def test_linear_refusals(lib):
    ok = dict(a=F, lda=256, ac=None, asc=None, wc=G, wsc=G + (1 << 24), bias=None, gate=None, out=H, ldo=64, M=40, N=64,
              K=256, epi=0, ws=I, wsb=1 << 20)

    def call(**kw):
        a = dict(ok, **kw)
        return lib.regenvc_mx_linear_fwd(*[a[n] for n in ("a", "lda", "ac", "asc", "wc", "wsc", "bias", "gate", "out", "ldo",
                                                          "M", "N", "K", "epi", "ws", "wsb")], None)
    refused(lib, INV, "negative", call(M=-1))
    refused(lib, INV, "epilogue", call(epi=3))
    refused(lib, INV, "gate needs", call(gate=I + 4096))
    refused(lib, UNS, "multiple of 16", call(N=72, ldo=72))
    refused(lib, UNS, "multiple of 8", call(K=252))
    refused(lib, UNS, "lda", call(lda=248))
    refused(lib, UNS, "lda", call(lda=260))
    refused(lib, UNS, "ldo", call(ldo=56))
    refused(lib, UNS, "ldo", call(ldo=68))
    refused(lib, UNS, "an output of", call(N=1 << 20, ldo=1 << 20))
    refused(lib, UNS, "rows, must be below", call(M=1 << 26))
    refused(lib, UNS, "an output of", call(M=1 << 30, N=1 << 14, ldo=1 << 14))
    refused(lib, INV, "give a, or", call(ac=F))
    refused(lib, INV, "NULL", call(a=None, ac=F))
    refused(lib, INV, "NULL", call(wc=None))
    refused(lib, INV, "NULL", call(out=None))
    refused(lib, UNS, "16-byte", call(a=F + 2))
    refused(lib, UNS, "16-byte", call(wsc=G + (1 << 24) + 8))
    refused(lib, UNS, "256-byte", call(ws=I + 128))
    refused(lib, INV, "out overlaps", call(out=F + 512))
    refused(lib, INV, "workspace overlaps", call(ws=G))
    refused(lib, INV, "workspace overlaps", call(ws=H))
    refused(lib, INV, "workspace_bytes", call(wsb=-1))
    assert call(M=0) == 0 and call(N=0, ldo=8) == 0
    n = ctypes.c_int64()
    need = lib.regenvc_mx_linear_workspace
    refused(lib, INV, "NULL", need(4, 16, 64, 0, None))
    refused(lib, UNS, "multiple of 16", need(4, 17, 64, 0, ctypes.byref(n)))


def cache(**kw):
    a = dict(dict(k=F, ks=G, v=H, vs=I, B=2, cap=100, heads=3, D=128), **kw)
    return ctypes.byref(_lib.MxCache(a["k"], a["ks"], a["v"], a["vs"], a["B"], a["cap"], a["heads"], a["D"]))


def view(ptr, S, heads, D, B=2):
    return ctypes.byref(_lib.Tensor(ptr, S * heads * D, heads * D, D))


T1, T2, T3 = F + (1 << 35), F + (1 << 36), F + (1 << 37)


def test_append_refusals(lib):
    k, v = view(T1, 5, 3, 128), view(T2, 5, 3, 128)

    def call(c=None, k=k, v=v, S=5, start=None, count=None):
        return lib.regenvc_mx_cache_append(c if c is not None else cache(), k, v, S, start, count, None)
    refused(lib, INV, "negative cache", call(cache(B=-1)))
    refused(lib, UNS, "D=96", call(cache(D=96)))
    refused(lib, INV, "NULL cache", call(cache(ks=None)))
    refused(lib, UNS, "codes are not 16", call(cache(v=H + 8)))
    refused(lib, INV, "S=-1", call(S=-1))
    refused(lib, INV, "k: data pointer", call(k=view(None, 5, 3, 128)))
    refused(lib, UNS, "stride_s", call(k=ctypes.byref(_lib.Tensor(T1, 1920, 388, 128))))
    refused(lib, INV, "overlaps", call(k=view(F, 5, 3, 128)))
    refused(lib, INV, "overlaps", call(cache(vs=F)))
    refused(lib, UNS, "4-byte", call(start=T3 + 2))
    refused(lib, INV, "overlaps", call(start=I))
    refused(lib, UNS, "a capacity of", call(cache(cap=(1 << 30) + 1)))
    refused(lib, INV, "cache is NULL", lib.regenvc_mx_cache_append(None, k, v, 5, None, None, None))
    assert call(S=0) == 0 and call(cache(B=0, k=None, ks=None, v=None, vs=None)) == 0
    refused(lib, INV, "overlap", lib.regenvc_mx_cache_values(cache(), T1, T1, 1, None))
    refused(lib, INV, "overlap", lib.regenvc_mx_cache_values(cache(), F, T1, 1, None))
    refused(lib, INV, "dtype", lib.regenvc_mx_cache_values(cache(), T2, T1, 5, None))
    refused(lib, INV, "NULL", lib.regenvc_mx_cache_values(cache(), None, T1, 0, None))


def test_attention_refusals(lib):
    q, o = view(T1, 7, 6, 128), view(T2, 7, 6, 128)
    ok = dict(q=q, c=cache(), lens=None, n=100, o=o, t=0, lse=T3, B=2, H=6, S=7, scale=0.1, ws=T3 + (1 << 30), wsb=1 << 28)

    def call(**kw):
        a = dict(ok, **kw)
        return lib.regenvc_mx_attn_cache_fwd(*[a[n] for n in ("q", "c", "lens", "n", "o", "t", "lse", "B", "H", "S", "scale",
                                                              "ws", "wsb")], None)
    refused(lib, INV, "negative", call(S=-1))
    refused(lib, INV, "multiple of the cache", call(H=7))
    refused(lib, INV, "sequences", call(B=3))
    refused(lib, INV, "max_len", call(n=101))
    refused(lib, INV, "negative", call(n=-1))
    refused(lib, INV, "dtype", call(t=3))
    refused(lib, INV, "softmax_scale", call(scale=-1.0))
    refused(lib, INV, "softmax_scale", call(scale=float("nan")))
    refused(lib, UNS, "D=32", call(c=cache(D=32)))
    refused(lib, INV, "q: data pointer", call(q=view(None, 7, 6, 128)))
    refused(lib, UNS, "16-byte", call(q=view(T1 + 8, 7, 6, 128)))
    refused(lib, INV, "share an address", call(o=ctypes.byref(_lib.Tensor(T2, 0, 768, 128))))
    refused(lib, INV, "overlaps an input", call(o=view(T1, 7, 6, 128)))
    refused(lib, INV, "overlaps an input", call(lse=G))
    refused(lib, INV, "overlaps an input", call(lens=T2))
    refused(lib, INV, "overlap", call(lse=T2))
    refused(lib, INV, "overlap", call(ws=T2))
    refused(lib, UNS, "256-byte", call(ws=T3 + (1 << 30) + 16))
    refused(lib, UNS, "4-byte", call(lens=T3 + (1 << 29) + 1))
    refused(lib, INV, "workspace_bytes", call(wsb=-1))
    assert call(S=0) == 0 and call(H=0) == 0


def test_attention_plans(lib):
    p, b = _lib.MxAttnPlan(), ctypes.c_int64()
    for B, H, heads, Sq, n, D in [(1, 12, 12, 1, 10920, 128), (1, 12, 12, 1560, 32760, 128), (16, 16, 4, 3, 10920, 64),
                                  (1, 1, 1, 1, 0, 64), (300, 12, 12, 1, 4000, 128), (1, 5, 1, 13, 100, 64),
                                  (2, 2, 2, 65, 1 << 20, 128)]:
        assert lib.regenvc_mx_attn_cache_plan_query(B, H, heads, Sq, n, D, 256, ctypes.byref(p)) == 0
        assert lib.regenvc_mx_attn_cache_workspace(B, H, heads, Sq, n, D, 256, ctypes.byref(b)) == 0
        rows = Sq * H // heads
        assert p.tile_rows * p.row_tiles >= rows > p.tile_rows * (p.row_tiles - 1) and 1 <= p.key_ranges <= 64
        assert b.value == (p.key_ranges * B * Sq * H * (D + 1) * 4 if p.key_ranges > 1 else 0)
    refused(lib, INV, "n_cu", lib.regenvc_mx_attn_cache_plan_query(1, 1, 1, 1, 1, 64, 0, ctypes.byref(p)))
    refused(lib, INV, "NULL", lib.regenvc_mx_attn_cache_plan_query(1, 1, 1, 1, 1, 64, 256, None))
    refused(lib, INV, "multiple", lib.regenvc_mx_attn_cache_workspace(1, 3, 2, 1, 1, 64, 256, ctypes.byref(b)))
    refused(lib, UNS, "2^29", lib.regenvc_mx_attn_cache_workspace(1 << 12, 1 << 10, 1, 1 << 10, 1, 64, 256, ctypes.byref(b)))
    refused(lib, UNS, "2^22", lib.regenvc_mx_attn_cache_workspace(1 << 20, 4, 4, 1, 1, 64, 256, ctypes.byref(b)))
    refused(lib, UNS, "max_len", lib.regenvc_mx_attn_cache_workspace(1, 1, 1, 1, (1 << 30) + 1, 64, 256, ctypes.byref(b)))


def test_linear_plans(lib):
    p, n, c, sc = _lib.TilePlan(), ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    for M, N, K, epi in [(1, 16, 8, 0), (64, 1536, 8960, 1), (65, 16, 8, 2), (1365, 1536, 8960, 0), (10920, 8960, 1536, 1),
                         (200, 8960, 8960, 2), (65520, 1536, 1536, 0)]:
        assert lib.regenvc_mx_linear_plan_query(M, N, K, epi, 256, ctypes.byref(p)) == 0
        assert p.k_ranges == 1 and p.rows >= 16 and p.cols >= 16 and p.waves in (4, 16)
        assert lib.regenvc_mx_linear_workspace(M, N, K, 1, ctypes.byref(n)) == 0 and n.value == 0
        assert lib.regenvc_mx_linear_workspace(M, N, K, 0, ctypes.byref(n)) == 0
        assert lib.regenvc_mx_bytes(M, K, ctypes.byref(c), ctypes.byref(sc)) == 0
        assert n.value == 0 if M <= 16 else n.value == 0 or n.value >= c.value + sc.value
    refused(lib, INV, "NULL", lib.regenvc_mx_linear_plan_query(4, 16, 64, 0, 256, None))
    refused(lib, INV, "n_cu", lib.regenvc_mx_linear_plan_query(4, 16, 64, 0, 0, ctypes.byref(p)))
    refused(lib, INV, "epilogue", lib.regenvc_mx_linear_plan_query(4, 16, 64, 7, 256, ctypes.byref(p)))


def test_residual_norm_refusals(lib):
    LN, RMS, NONE = (_lib.Norm(k, 1e-6, None, None) for k in (1, 2, 0))
    none = _lib.RowVectors(None, None, None, 64, 0)
    ok = dict(x=F, ldx=64, y=G, ldy=64, t=0, post=NONE, pre=LN, v=none, alpha=1.0, xo=H, ldxo=64, h=I, ldh=64, rows=10, C=64)

    def fwd(**kw):
        a = dict(ok, **kw)
        return lib.regenvc_residual_norm_fwd(a["x"], a["ldx"], a["y"], a["ldy"], a["t"], a["post"], a["pre"], a["v"],
                                             a["alpha"], a["xo"], a["ldxo"], a["h"], a["ldh"], a["rows"], a["C"], None)
    refused(lib, INV, "rows=-1", fwd(rows=-1))
    refused(lib, UNS, "must be below", fwd(rows=1 << 26))
    refused(lib, UNS, "must be below", fwd(rows=1 << 24, C=4096))
    for C in (0, 12, 8200):
        refused(lib, UNS, "multiple of 8", fwd(C=C))
    refused(lib, INV, "dtype", fwd(t=9))
    refused(lib, INV, "pre kind", fwd(pre=NONE))
    refused(lib, INV, "post kind", fwd(post=_lib.Norm(5, 1e-6, None, None)))
    refused(lib, INV, "eps", fwd(pre=_lib.Norm(1, -1.0, None, None)))
    refused(lib, INV, "eps", fwd(post=_lib.Norm(1, float("nan"), None, None)))
    refused(lib, INV, "no bias", fwd(pre=_lib.Norm(2, 1e-6, T1, T1)))
    refused(lib, INV, "no norm", fwd(post=_lib.Norm(0, 1e-6, T1, None)))
    refused(lib, INV, "alpha", fwd(alpha=float("inf")))
    refused(lib, INV, "vectors is NULL", fwd(v=None))
    refused(lib, INV, "group_rows", fwd(v=_lib.RowVectors(None, None, None, 64, -1)))
    refused(lib, INV, "together", fwd(v=_lib.RowVectors(None, T1, None, 64, 0)))
    refused(lib, INV, "or the weights", fwd(v=_lib.RowVectors(None, T1, T1, 64, 0), pre=_lib.Norm(1, 1e-6, T2, None)))
    refused(lib, UNS, "elements apart", fwd(v=_lib.RowVectors(T1, None, None, 60, 3)))
    refused(lib, UNS, "elements apart", fwd(v=_lib.RowVectors(T1, None, None, 66, 3)))
    for ld in ("ldx", "ldy", "ldxo", "ldh"):
        refused(lib, UNS, ld, fwd(**{ld: 56}))
        refused(lib, UNS, ld, fwd(**{ld: 68}))
    for p in ("x", "y", "xo", "h"):
        refused(lib, INV, "NULL", fwd(**{p: None}))
        refused(lib, UNS, "16-byte", fwd(**{p: ok[p] + 8}))
    refused(lib, UNS, "gate is not", fwd(v=_lib.RowVectors(T1 + 4, None, None, 64, 0)))
    refused(lib, INV, "h overlaps x", fwd(h=F))
    refused(lib, INV, "x_out overlaps x", fwd(xo=F + 256))
    refused(lib, INV, "x_out overlaps x", fwd(xo=F, ldxo=72))
    refused(lib, INV, "x_out overlaps h", fwd(xo=I))
    refused(lib, INV, "overlaps y", fwd(xo=G))
    assert fwd(rows=0) == 0
    bk = dict(x=F, y=G, t=0, post=NONE, pre=LN, v=none, alpha=1.0, gh=H, gx=None, dx=I, dy=T1, g=_lib.NormGrads(), rows=10,
              C=64, ws=None, wsb=0)

    def bwd(**kw):
        a = dict(bk, **kw)
        return lib.regenvc_residual_norm_bwd(a["x"], 64, a["y"], 64, a["t"], a["post"], a["pre"], a["v"], a["alpha"],
                                             a["gh"], 64, a["gx"], 64, a["dx"], 64, a["dy"], 64, a["g"], a["rows"], a["C"],
                                             a["ws"], a["wsb"], None)
    for n in _lib.NORM_GRAD_NAMES:
        refused(lib, INV, "not there", bwd(g=_lib.NormGrads(**{n: T2})))
    refused(lib, INV, "grads is NULL", bwd(g=None))
    refused(lib, INV, "together", bwd(v=_lib.RowVectors(None, None, T2, 64, 0)))
    refused(lib, INV, "NULL data", bwd(gh=None))
    refused(lib, INV, "dx overlaps x_out", bwd(dx=F))
    refused(lib, INV, "dy overlaps gh", bwd(dy=H))
    refused(lib, INV, "dx overlaps dy", bwd(dx=T1))
    refused(lib, INV, "workspace overlaps", bwd(ws=G, wsb=256))
    refused(lib, UNS, "256-byte", bwd(ws=T3 + 16, wsb=256))
    refused(lib, INV, "workspace_bytes", bwd(wsb=-1))
    one = _lib.RowVectors(T2, None, None, 64, 0)
    refused(lib, INV, "dgate overlaps gate", bwd(v=one, g=_lib.NormGrads(dgate=T2)))
    refused(lib, INV, "at least one row", bwd(rows=0, pre=_lib.Norm(1, 1e-6, T2, None), g=_lib.NormGrads(dw=T3)))
    assert bwd(rows=0) == 0
    n = ctypes.c_int64()
    need = lib.regenvc_residual_norm_bwd_workspace
    refused(lib, INV, "bad size", need(4, 64, 0, 4, 0, 256, ctypes.byref(n)))
    refused(lib, INV, "NULL", need(4, 64, 0, 1, 0, 256, None))
    refused(lib, UNS, "multiple of 8", need(4, 65, 0, 1, 0, 256, ctypes.byref(n)))
    assert need(0, 64, 0, 3, 4, 256, ctypes.byref(n)) == 0 and n.value == 0
    assert need(10, 64, 1, 3, 0, 256, ctypes.byref(n)) == 0 and n.value == 0
    assert need(10920, 1536, 1560, 3, 2, 256, ctypes.byref(n)) == 0 and 0 < n.value < 1 << 26
