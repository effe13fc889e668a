"""Sizes beyond 32 bits in the torch binding of the residual norm and the MXFP4
calls, on the CPU: the library is replaced by one that notes what it is handed,
and host tensors pass for device tensors.  A size never reaches it as its low 32
bits (a group of 2^32 + 1 rows as one of 1 row, whose vectors are not there)."""
import contextlib
import sys

import pytest

from paper_2607_28144_amd import _lib

torch = pytest.importorskip("torch")

WIDE = (1 << 31, (1 << 32) + 1, (1 << 33) + 5)


class Recorder:
    """Notes the group_rows and the rows of the seam's calls, and calls of any other name."""

    def __init__(self):
        self.seen = []

    def regenvc_residual_norm_fwd(self, *a):
        self.seen.append((a[7]._obj.group_rows, a[13]))
        return _lib.OK

    def regenvc_residual_norm_bwd(self, *a):
        self.seen.append((a[7]._obj.group_rows, a[18]))
        return _lib.OK

    def regenvc_residual_norm_bwd_workspace(self, rows, C, group_rows, group_sums, row_sums, n_cu, out):
        self.seen.append((group_rows, rows))
        out._obj.value = 0
        return _lib.OK

    def __getattr__(self, name):
        def call(*a):
            self.seen.append(name)
            return _lib.OK
        return call


@pytest.fixture
def lib(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(_lib, "load", lambda: r)
    monkeypatch.setattr(_lib, "index_of", lambda t, name: -1)  # as get_device() of a host tensor
    monkeypatch.setattr(_lib, "on_device", lambda idx: contextlib.nullcontext())
    monkeypatch.setattr(_lib, "raw_stream", lambda idx: 0)
    monkeypatch.setattr(_lib, "compute_units", lambda idx: 256)
    return r


def seam(group_rows):
    from paper_2607_28144_amd import dit
    x, y = torch.zeros(10, 64), torch.zeros(10, 64, dtype=torch.bfloat16)
    gate = torch.zeros(-(-10 // group_rows) if 0 < group_rows < 10 else 1, 64)
    dit.residual_norm_fwd(x, y, gate=gate, group_rows=group_rows)
    g = dit.residual_norm_bwd(x, y, y, gate=gate, group_rows=group_rows)
    return g.dgate.shape[0]


@pytest.mark.parametrize("group_rows", [10, 11, (1 << 31) - 1, *WIDE, sys.maxsize])
def test_a_group_of_all_rows_or_more_is_one_set(lib, group_rows):
    assert seam(group_rows) == 1
    assert lib.seen and all(gr >= n == 10 for gr, n in lib.seen)


def test_groups_within_the_rows_are_handed_on(lib):
    for group_rows, groups in ((0, 1), (1, 10), (3, 4), (9, 2), (-1, 1)):
        lib.seen.clear()
        assert seam(group_rows) == groups
        assert lib.seen and all(s == (group_rows, 10) for s in lib.seen)


@pytest.mark.parametrize("group_rows", [-(1 << 31) - 1, -(1 << 32) + 1])
def test_a_negative_group_stays_negative(lib, group_rows):
    with pytest.raises(ValueError, match="group_rows"):
        seam(group_rows)
    assert not lib.seen


@pytest.mark.parametrize("n", [*WIDE, -(1 << 31) - 1])
def test_mxfp4_sizes(lib, n):
    """Matrices, caches, appended tokens (a broadcast view has as many as one likes) and planned lengths."""
    from paper_2607_28144_amd import mx
    for sizes in ((n, 64), (64, n)):
        with pytest.raises(ValueError, match="32 bits"):
            mx.mx_bytes(*sizes)
        with pytest.raises(ValueError, match="32 bits"):
            mx.linear_workspace_bytes(16, *sizes, True)
    with pytest.raises(ValueError, match="32 bits"):
        mx.linear_workspace_bytes(n, 16, 64, True)
    for sizes in ((n, 0, 1), (1, n, 0), (0, 1, n)):
        with pytest.raises(ValueError, match="32 bits"):
            mx.KvCache(*sizes, 64)
    cache = object.__new__(mx.KvCache)
    cache.batch, cache.capacity, cache.heads, cache.D = 1, 8, 1, 64
    cache.device = torch.device("cuda", 0)
    if n > 0:
        k = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16).expand(1, n, 1, 64)
        with pytest.raises(ValueError, match="32 bits"):
            cache.append(k, k)
    with pytest.raises(ValueError, match="32 bits"):
        mx._attn_need(1, 1, 1, 1, n, 64, 0)
    assert not lib.seen
