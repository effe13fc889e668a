"""Host side of include/regenvc_paged.h and of its binding on the CPU: bad
arguments are refused before any HIP call (the fake addresses are never
dereferenced), and the plans are sound."""
import contextlib
import ctypes
import os
import re

import pytest

from conftest import REPO
from paper_2607_28144_amd import _lib

A = 0x10000000    # 256-byte aligned, never dereferenced; each region has 2^32 bytes
K, V, M, Q, KN, VN, O, L, TAB, FIRST, LENS, WS, SEL, WT = (A + (i << 32) for i in range(14))
INV, UNS = _lib.ERR_INVALID_ARG, _lib.ERR_UNSUPPORTED
ref = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def refused(lib, status, word, st):
    assert st == status, (st, lib.regenvc_last_error())
    assert word in lib.regenvc_last_error().decode(), lib.regenvc_last_error()


def pool(**kw):
    a = dict(dict(k=K, v=V, means=M, pages=10, page=64, heads=2, D=128), **kw)
    return _lib.PagePool(*a.values())


def batch(**kw):
    a = dict(dict(table=TAB, first=FIRST, lens=LENS, table_stride=5, B=2, columns=5, T=7), **kw)
    return _lib.PageBatch(*a.values())


def view(ptr, heads, D=128):
    return _lib.Tensor(ptr, 0, heads * D, D)


def test_every_declared_symbol_is_bound(lib):
    text = open(os.path.join(REPO, "include", "regenvc_paged.h")).read()
    names = set(re.findall(r"^regenvc_status\s+(regenvc_\w+)\s*\(", text, re.M))
    assert len(names) == 5
    for n in names:
        assert hasattr(lib, n) and n in _lib._SIGNATURES


BAD_POOLS = [(INV, "negative", dict(pages=-1)), (INV, "negative", dict(heads=-1)), (UNS, "D=", dict(D=96)),
             (UNS, "places", dict(page=48)), (UNS, "places", dict(page=8)), (UNS, "places", dict(page=2048)),
             (UNS, "places", dict(page=-16)), (UNS, "pages of", dict(pages=1 << 30)), (UNS, "heads", dict(heads=65536)),
             (INV, "NULL", dict(k=None)), (INV, "NULL", dict(v=None)), (UNS, "16-byte", dict(k=K + 8)),
             (UNS, "16-byte", dict(means=M + 2))]
BAD_BATCHES = [(INV, "negative", dict(B=-1)), (INV, "negative", dict(T=-1)), (INV, "negative", dict(columns=-1)),
               (UNS, "too many", dict(B=(1 << 20) + 1)), (UNS, "too many", dict(T=1 << 26)),
               (UNS, "too many", dict(columns=1 << 24)), (INV, "NULL", dict(table=None)), (INV, "NULL", dict(first=None)),
               (INV, "NULL", dict(lens=None)), (UNS, "4-byte", dict(lens=LENS + 2)), (UNS, "table_stride", dict(table_stride=-1)),
               (UNS, "table_stride", dict(table_stride=1 << 40))]


def test_append_refusals(lib):
    def call(p=None, n=None, q=view(Q, 4), k=view(KN, 2), v=view(VN, 2), wq=WT, wk=WT + 256, eps=1e-6, rot=(WT + 512, 64, 0, 1.0),
             out=view(O, 4), H=4):
        by = lambda x: None if x is None else ref(x)  # noqa: E731
        return lib.regenvc_paged_append(by(pool() if p is None else p), by(batch() if n is None else n), by(q), by(k), by(v), wq,
                                        wk, eps, None if rot is None else ref(_lib.RotaryTable(*rot)), by(out), H, None)
    for st, word, kw in BAD_POOLS:
        refused(lib, st, word, call(p=pool(**kw)))
    for st, word, kw in BAD_BATCHES:
        refused(lib, st, word, call(n=batch(**kw)))
    refused(lib, INV, "pool is NULL", lib.regenvc_paged_append(None, ref(batch()), None, None, None, None, None, 0.0, None, None, 0,
                                                               None))
    refused(lib, INV, "batch is NULL", lib.regenvc_paged_append(ref(pool()), None, None, None, None, None, None, 0.0, None, None, 0,
                                                                None))
    refused(lib, INV, "go together", call(q=None))
    refused(lib, INV, "go together", call(out=None))
    refused(lib, INV, "go together", call(H=0))
    refused(lib, INV, "go together", call(q=None, out=None, H=0))  # w_q without q
    refused(lib, INV, "H=-1", call(H=-1))
    refused(lib, INV, "eps", call(eps=-1.0))
    refused(lib, INV, "eps", call(eps=float("nan")))
    refused(lib, INV, "eps", call(eps=float("inf")))
    refused(lib, UNS, "pairs", call(rot=(WT + 512, 72, 0, 1.0)))
    refused(lib, UNS, "pairs", call(rot=(WT + 512, 4, 0, 1.0)))
    refused(lib, UNS, "pairs", call(rot=(WT + 512, -8, 0, 1.0)))
    refused(lib, INV, "turns", call(rot=(None, 64, 0, 1.0)))
    refused(lib, UNS, "turns", call(rot=(WT + 516, 64, 0, 1.0)))
    refused(lib, INV, "amplitude", call(rot=(WT + 512, 64, 0, float("inf"))))
    refused(lib, UNS, "w_q", call(wq=WT + 8))
    refused(lib, INV, "NULL", call(k=None))
    refused(lib, INV, "NULL", call(v=view(None, 2)))
    refused(lib, UNS, "aligned", call(q=view(Q + 2, 4)))
    refused(lib, UNS, "multiple of 8", call(k=_lib.Tensor(KN, 0, 260, 128)))
    refused(lib, INV, "share an address", call(out=_lib.Tensor(O, 0, 128, 128)))
    refused(lib, INV, "pool overlaps itself", call(p=pool(v=K + 256)))
    refused(lib, INV, "pool overlaps another", call(k=view(V + 1024, 2)))
    refused(lib, INV, "pool overlaps another", call(n=batch(lens=M + 64)))
    refused(lib, INV, "pool overlaps another", call(out=view(K, 4)))
    refused(lib, INV, "q_out overlaps", call(out=view(Q + 256, 4)))
    refused(lib, INV, "q_out overlaps", call(out=view(KN, 4)))
    refused(lib, INV, "q_out overlaps", call(out=view(WT, 4)))
    # within a fused projection: q_out may be q's part, and not one that reaches into k's
    fused = lambda at, heads: _lib.Tensor(Q + at * 256, 0, 8 * 128, 128)  # noqa: E731
    refused(lib, INV, "q_out overlaps", call(q=fused(0, 4), k=fused(4, 2), v=fused(6, 2), out=fused(1, 4)))
    refused(lib, INV, "q_out overlaps", call(q=fused(0, 4), k=fused(3, 2), v=fused(6, 2), out=fused(0, 4)))
    assert call(n=batch(B=0)) == 0 and call(n=batch(T=0)) == 0
    assert call(p=pool(heads=0), q=None, out=None, H=0, wq=None) == 0


def test_select_refusals(lib):
    def call(p=None, n=None, q=view(Q, 4), H=4, q_block=2, count=3, kf=1, kl=1, sel=SEL):
        return lib.regenvc_paged_select(None if q is None else ref(q), ref(pool() if p is None else p),
                                        ref(batch() if n is None else n), H, q_block, count, kf, kl, 1, sel, None)
    for st, word, kw in BAD_POOLS:
        refused(lib, st, word, call(p=pool(**kw)))
    for st, word, kw in BAD_BATCHES:
        refused(lib, st, word, call(n=batch(**kw)))
    refused(lib, UNS, "multiple", call(H=3))
    refused(lib, INV, "H=", call(H=-2))
    refused(lib, UNS, "multiple", call(p=pool(heads=0)))
    for kw in ({"q_block": 0}, {"q_block": (1 << 20) + 1}, {"count": 0}, {"count": 16385}):
        refused(lib, UNS, "q_block", call(**kw))
    refused(lib, INV, "keep_first", call(kf=2, kl=2))
    refused(lib, INV, "keep_first", call(kf=-1))
    refused(lib, INV, "keep_first", call(kl=-1))
    refused(lib, INV, "keep_first", call(kf=(1 << 31) - 1, kl=(1 << 31) - 1))
    refused(lib, UNS, "columns", call(n=batch(columns=16385)))
    refused(lib, UNS, "blocks", call(n=batch(T=(1 << 26) - 1), q_block=1))
    refused(lib, INV, "means", call(p=pool(means=None)))
    refused(lib, INV, "NULL", call(q=None))
    refused(lib, INV, "selected is NULL", call(sel=None))
    refused(lib, UNS, "4-byte", call(sel=SEL + 2))
    refused(lib, INV, "overlaps", call(sel=Q + 16))
    refused(lib, INV, "overlaps", call(sel=M))
    refused(lib, INV, "overlaps", call(sel=TAB))
    # without a query there are blocks all the same, and entries to write; none with neither rows nor sequences
    for kw in ({"n": batch(T=0)}, {"n": batch(B=0)}, {"H": 0}):
        refused(lib, INV, "selected is NULL", call(sel=None, q=None, **kw))
    assert call(n=batch(B=0, T=1)) == 0 and call(n=batch(B=0, T=0)) == 0


def test_attention_refusals(lib):
    def call(p=None, n=None, q=view(Q, 4), sel=None, q_block=1, count=0, rows=7, places=320, o=view(O, 4), dt=0, lse=L, H=4,
             scale=0.1, ws=WS, wsb=1 << 20):
        return lib.regenvc_paged_attn_fwd(None if q is None else ref(q), ref(pool() if p is None else p),
                                          ref(batch() if n is None else n), sel, q_block, count, 1, rows, places,
                                          None if o is None else ref(o), dt, lse, H, scale, ws, wsb, None)
    for st, word, kw in BAD_POOLS:
        refused(lib, st, word, call(p=pool(**kw)))
    for st, word, kw in BAD_BATCHES:
        refused(lib, st, word, call(n=batch(**kw)))
    refused(lib, UNS, "multiple", call(H=3))
    refused(lib, UNS, "q_block", call(sel=SEL, count=0))
    refused(lib, UNS, "q_block", call(sel=SEL, count=4, q_block=0))
    refused(lib, INV, "max_rows", call(rows=8))
    refused(lib, INV, "negative", call(rows=-1))
    refused(lib, INV, "max_len", call(places=321))
    refused(lib, INV, "negative", call(places=-1))
    refused(lib, UNS, "rows, at most", call(n=batch(T=(1 << 26) - 1), H=16, rows=1))
    refused(lib, INV, "scale", call(scale=-1.0))
    refused(lib, INV, "scale", call(scale=float("nan")))
    refused(lib, INV, "dtype", call(dt=3))
    refused(lib, INV, "NULL", call(q=None))
    refused(lib, INV, "NULL", call(o=None))
    refused(lib, INV, "share an address", call(o=_lib.Tensor(O, 0, 128, 128)))
    refused(lib, UNS, "4-byte", call(lse=L + 1))
    refused(lib, UNS, "4-byte", call(sel=SEL + 2, count=4))
    refused(lib, UNS, "256-byte", call(ws=WS + 16))
    refused(lib, INV, "workspace_bytes", call(wsb=-1))
    refused(lib, INV, "overlaps an input", call(o=view(Q, 4)))
    refused(lib, INV, "overlaps an input", call(lse=K + 4))
    refused(lib, INV, "overlaps an input", call(ws=FIRST))
    refused(lib, INV, "overlaps an input", call(sel=SEL, count=4, lse=SEL + 4))
    refused(lib, INV, "o, lse and the workspace", call(lse=O + 64))
    refused(lib, INV, "o, lse and the workspace", call(ws=O))
    assert call(n=batch(B=0)) == 0 and call(n=batch(T=0), rows=0) == 0 and call(H=0) == 0


def shape(**kw):
    a = dict(dict(B=1, T=1, H=12, heads=12, D=128, page=64, q_block=1, count=0, max_rows=1, max_len=32760), **kw)
    return _lib.PagedAttnShape(*a.values())


def test_plans(lib):
    p, n = _lib.PagedAttnPlan(), ctypes.c_int64()
    refused(lib, INV, "NULL", lib.regenvc_paged_attn_plan_query(ref(shape()), 256, None))
    refused(lib, INV, "NULL", lib.regenvc_paged_attn_plan_query(None, 256, ref(p)))
    refused(lib, INV, "n_cu", lib.regenvc_paged_attn_plan_query(ref(shape()), 0, ref(p)))
    refused(lib, INV, "NULL", lib.regenvc_paged_attn_workspace(ref(shape()), 256, None))
    refused(lib, INV, "n_cu", lib.regenvc_paged_attn_workspace(ref(shape()), 0, ref(n)))
    refused(lib, UNS, "D=", lib.regenvc_paged_attn_workspace(ref(shape(D=96)), 256, ref(n)))
    refused(lib, UNS, "places", lib.regenvc_paged_attn_workspace(ref(shape(page=20)), 256, ref(n)))
    refused(lib, UNS, "too many", lib.regenvc_paged_attn_workspace(ref(shape(max_len=1 << 30)), 256, ref(n)))
    refused(lib, INV, "max_rows", lib.regenvc_paged_attn_workspace(ref(shape(max_rows=2)), 256, ref(n)))
    refused(lib, INV, "negative", lib.regenvc_paged_attn_workspace(ref(shape(B=-1)), 256, ref(n)))
    refused(lib, UNS, "workgroups", lib.regenvc_paged_attn_workspace(ref(shape(T=(1 << 26) - 1, H=2, heads=2, count=1)), 256,
                                                                     ref(n)))
    for kw in (dict(), dict(B=16, T=16, H=16, heads=4, D=64), dict(T=10920, max_rows=10920), dict(T=77, max_rows=40, B=3),
               dict(H=40, heads=1), dict(T=1560, max_rows=1560, q_block=64, count=64), dict(B=5, T=5, q_block=1, count=16),
               dict(T=0, max_rows=0), dict(B=0), dict(H=0), dict(max_len=0), dict(T=9, max_rows=0)):
        for n_cu in (1, 64, 256):
            s = shape(**kw)
            assert lib.regenvc_paged_attn_plan_query(ref(s), n_cu, ref(p)) == 0
            assert lib.regenvc_paged_attn_workspace(ref(s), n_cu, ref(n)) == 0
            if s.B * s.T * s.H == 0:
                assert p.tile_rows == p.workgroups == p.split == 0 and n.value == 0
                continue
            assert p.tile_rows in (16, 32, 64, 256) and p.workgroups >= s.heads
            assert n.value == (4 * (p.workgroups * p.tile_rows * (s.D + 1) + 2 * s.T * s.H) if p.split else 0)


torch = pytest.importorskip("torch")


@pytest.fixture
def host(monkeypatch):
    """Host tensors pass for device tensors, and the library notes what it is handed."""
    class Recorder:
        seen = []

        def __getattr__(self, name):
            def call(*a):
                self.seen.append(name)
                return _lib.OK
            return call
    r = Recorder()
    r.seen = []
    monkeypatch.setattr(_lib, "load", lambda: r)
    monkeypatch.setattr(_lib, "index_of", lambda t, name: -1)
    monkeypatch.setattr(_lib, "on_device", lambda idx: contextlib.nullcontext())
    monkeypatch.setattr(_lib, "raw_stream", lambda idx: 0)
    monkeypatch.setattr(_lib, "compute_units", lambda idx: 256)
    from paper_2607_28144_amd import paged
    monkeypatch.setattr(paged, "_index", lambda cache: -1)
    return r


def bf(*s):
    return torch.zeros(*s, dtype=torch.bfloat16)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_binding_refusals(host):
    from paper_2607_28144_amd import paged
    c = paged.PagedCache(bf(6, 2, 16, 64), bf(6, 2, 16, 64), bf(6, 2, 64))
    seqs = dict(table=torch.zeros(2, 3, dtype=torch.int32), first=i32(0, 1, 3), lens=i32(5, 9))
    q, k = bf(3, 4, 64), bf(3, 2, 64)
    paged.attn_fwd(q, c, **seqs)
    paged.attn_pages_fwd(q, c, selected=torch.zeros(3, 2, 4, dtype=torch.int32), q_block=2, **seqs)
    paged.select_pages(q, c, count=2, q_block=2, **seqs)
    paged.append(c, k=k, v=k, q=q, **seqs)
    assert paged.append(c, k=k, v=k, **seqs) is None
    assert host.seen.count("regenvc_paged_attn_fwd") == 2 and host.seen.count("regenvc_paged_append") == 2
    n = len(host.seen)
    bad = [lambda: paged.PagedCache(bf(6, 2, 16, 64), bf(6, 2, 32, 64)), lambda: paged.PagedCache(bf(6, 2, 64), bf(6, 2, 64)),
           lambda: paged.PagedCache(bf(6, 2, 16, 64), bf(6, 2, 16, 64), bf(6, 64)),
           lambda: paged.PagedCache(bf(6, 2, 16, 64).float(), bf(6, 2, 16, 64).float()),
           lambda: paged.PagedCache(bf(6, 2, 16, 128)[..., :64], bf(6, 2, 16, 64)),
           lambda: paged.attn_fwd(bf(3, 4, 128), c, **seqs), lambda: paged.attn_fwd(bf(3, 64), c, **seqs),
           lambda: paged.attn_fwd(q.float(), c, **seqs), lambda: paged.attn_fwd(q, c, **dict(seqs, first=i32(0, 1))),
           lambda: paged.attn_fwd(q, c, **dict(seqs, lens=seqs["lens"].long())),
           lambda: paged.attn_fwd(q, c, **dict(seqs, table=torch.zeros(6, dtype=torch.int32))),
           lambda: paged.attn_fwd(q, c, out=bf(3, 2, 64), **seqs), lambda: paged.attn_fwd(q, c, lse_out=torch.zeros(3, 4), **seqs),
           lambda: paged.attn_fwd(q, c, max_len=1 << 32, **seqs), lambda: paged.attn_fwd(q, c, max_rows=1 << 33, **seqs),
           lambda: paged.attn_pages_fwd(q, c, selected=torch.zeros(2, 2, 4, dtype=torch.int32), q_block=2, **seqs),
           lambda: paged.attn_pages_fwd(q, c, selected=torch.zeros(3, 2, 4), q_block=2, **seqs),
           lambda: paged.attn_pages_fwd(q, c, selected=torch.zeros(3, 2, 4, dtype=torch.int32), q_block=0, **seqs),
           lambda: paged.attn_pages_fwd(q, c, selected=torch.zeros(3, 2, 4, dtype=torch.int32), q_block=(1 << 32) + 2, **seqs),
           lambda: paged.select_pages(q, c, count=1 << 32, **seqs), lambda: paged.select_pages(q, c, count=2, q_block=0, **seqs),
           lambda: paged.select_pages(q, c, count=2, out=torch.zeros(3, 2, 2, dtype=torch.int32), **seqs),
           lambda: paged.select_pages(q, c, count=2, keep_first=1 << 33, **seqs),
           lambda: paged.select_pages(q, paged.PagedCache(bf(6, 2, 16, 64), bf(6, 2, 16, 64)), count=2, **seqs),
           lambda: paged.append(c, k=k, v=bf(2, 2, 64), **seqs), lambda: paged.append(c, k=k, v=k, q_out=q, **seqs),
           lambda: paged.append(c, k=k, v=k, w_k=bf(128), **seqs), lambda: paged.append(c, k=k, v=k, q=q, q_out=bf(3, 4, 128), **seqs)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        paged.attn_fwd(q, c, out_dtype=torch.float16, **seqs)
    assert len(host.seen) == n
