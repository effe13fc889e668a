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
