"""Calls at and beyond the limits of the paged cache's entry points, on the CPU:
what a kernel could not do, or would read as another call, is refused."""
import ctypes

import pytest

from paper_2607_28144_amd import _lib
from test_paged_abi import bf, host, i32  # noqa: F401

torch = pytest.importorskip("torch")
ref = ctypes.byref


def test_attention_to_an_empty_list_of_pages(host):  # noqa: F811
    """A list without entries, or none at all, is not attention to every page."""
    from paper_2607_28144_amd import paged
    c = paged.PagedCache(bf(6, 2, 16, 64), bf(6, 2, 16, 64))
    seqs = dict(table=torch.zeros(2, 3, dtype=torch.int32), first=i32(0, 1, 3), lens=i32(5, 9))
    for selected in (torch.zeros(3, 2, 0, dtype=torch.int32), None):
        with pytest.raises(ValueError, match="selected"):
            paged.attn_pages_fwd(bf(3, 4, 64), c, selected=selected, q_block=2, **seqs)
    assert host.seen == []


def plan(**kw):
    """Status, tile rows and workgroups of the plan of a shape on 256 compute units."""
    a = dict(dict(B=1, T=1, H=1, heads=1, D=128, page=64, q_block=1, count=0, max_rows=1, max_len=64, causal=1), **kw)
    p, n = _lib.PagedAttnPlan(), ctypes.c_int64()
    lib = _lib.load()
    st = lib.regenvc_paged_attn_plan_query(ref(_lib.PagedAttnShape(*a.values())), 256, ref(p))
    assert st == lib.regenvc_paged_attn_workspace(ref(_lib.PagedAttnShape(*a.values())), 256, ref(n))
    return st, p.tile_rows, p.workgroups


# Calls just within what one launch can have (fewer than 2^32 threads), and just beyond: tile rows, threads, shape, what changes
LAUNCHES = [(16, 512, dict(H=8, heads=8, count=16), dict(T=(1 << 20) - 2), dict(T=(1 << 20) - 1)),
            (16, 512, dict(B=1 << 20, T=1 << 20), dict(H=7, heads=7), dict(H=8, heads=8)),
            (32, 256, dict(H=32, heads=2, q_block=2, count=16, max_rows=2), dict(T=(1 << 24) - 4), dict(T=(1 << 24) - 2)),
            (64, 256, dict(B=1 << 20, T=64, q_block=64, count=16, max_rows=64), dict(H=15, heads=15), dict(H=16, heads=16)),
            (256, 512, dict(B=1 << 20, T=300, q_block=300, count=16, max_rows=300), dict(H=3, heads=3), dict(H=4, heads=4))]


@pytest.mark.parametrize("rows,threads,shape,within,beyond", LAUNCHES)
def test_workgroups_of_one_launch(rows, threads, shape, within, beyond):
    st, tile, groups = plan(**shape, **within)
    assert st == _lib.OK and tile == rows and groups * threads < 1 << 32
    st, _, _ = plan(**shape, **beyond)
    assert st == _lib.ERR_UNSUPPORTED
    assert "workgroups" in _lib.load().regenvc_last_error().decode()


A = 0x10000000  # 256-byte aligned, never dereferenced
K, V, M, Q, TAB, FIRST, LENS, SEL = (A + (i << 44) for i in range(8))


def select(H, T, heads=1, q_block=1, pages=10, page=16, stride=0):
    pool = _lib.PagePool(K, V, M, pages, page, heads, 64)
    batch = _lib.PageBatch(TAB, FIRST, LENS, 5, 1, 5, T)
    q = _lib.Tensor(Q, 0, stride, stride)
    return _lib.load().regenvc_paged_select(ref(q), ref(pool), ref(batch), H, q_block, 2, 1, 1, 1, SEL, None)


@pytest.mark.parametrize("H,T,q_block", [(2048, 1 << 20, 1 << 20), (4096, 1 << 19, 1 << 19), (1 << 20, 1 << 10, 1 << 10),
                                         (513, 1 << 20, 1), (16, (1 << 26) - 1, 1 << 20)])
def test_choice_of_more_rows_than_32_bits_count(H, T, q_block):
    """A block's rows (queries times the heads that share a key head) are counted in 32 bits: H T is held to 2^29."""
    assert select(H, T, q_block=q_block) == _lib.ERR_UNSUPPORTED
    assert "rows, at most" in _lib.load().regenvc_last_error().decode()


@pytest.mark.parametrize("pages,heads,page", [((1 << 30) - 1, 65535, 1024), ((1 << 30) - 1, 128, 16), (1 << 26, 65535, 64),
                                              (1 << 20, 65535, 1024)])
def test_pool_of_more_bytes_than_there_are_addresses(pages, heads, page):
    """Its extent, which the checks of overlaps go by, would wrap."""
    assert select(heads, 3, heads, pages=pages, page=page, stride=64) == _lib.ERR_UNSUPPORTED
    assert "bytes" in _lib.load().regenvc_last_error().decode()


def test_keys_are_cut_up_to_256_sequences():
    """Single tokens against up to 4096 places: cut into ranges for up to 256 sequences, beyond them not."""
    def split(**kw):
        a = dict(dict(B=1, T=1, H=1, heads=1, D=64, page=64, q_block=1, count=0, max_rows=1, max_len=4096, causal=1), **kw)
        p = _lib.PagedAttnPlan()
        assert _lib.load().regenvc_paged_attn_plan_query(ref(_lib.PagedAttnShape(*a.values())), 256, ref(p)) == _lib.OK
        return p.split
    assert split(B=256, T=256) == 1 and split(B=257, T=257) == 0
    # of one sequence a short causal call has two rounds of workgroups: its tiles differ in their keys
    shape = dict(H=4, heads=4, page=64, T=600, max_rows=600, max_len=2112)
    assert plan(**shape, causal=1)[1:] == (256, 512) and plan(**shape, causal=0)[1:] == (256, 256)
    assert split(**dict(shape, causal=1)) == split(**dict(shape, causal=0)) == 1


@pytest.mark.parametrize("q_block,page", [(1, 16), (2, 16), (16, 16), (17, 16), (18, 16), (64, 64), (64, 16), (20, 128)])
def test_last_pages_that_keep_a_query_its_own(q_block, page):
    """In the definition of the choice: with ceil((q_block - 1) / page) + 1 last pages, and no fewer, the page of every query
    of a causal call is in its block's list, wherever the block begins."""
    import numpy as np

    from oracle import paged as opaged
    need = -(-(q_block - 1) // page) + 1
    pages = need + 4
    rows = pages * page
    # scores fall from page to page: none but the kept ones and the first few wins
    means = -np.arange(pages, dtype=np.float64)[:, None, None] * np.ones((1, 1, 64))
    q, table = np.ones((rows, 1, 64)), np.arange(pages)[None]

    def kept(keep_last, start):
        n = rows - start
        got = opaged.select(q[:n], means, table, [0, n], [rows], page, need, q_block, 0, keep_last, True)
        return all((start + t) // page in got[t // q_block, 0] for t in range(n))
    starts = range(page)
    assert all(kept(need, s) for s in starts)
    assert need == 1 or not all(kept(need - 1, s) for s in starts)
