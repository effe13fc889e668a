"""Argument checks of the residual-norm entry points (include/regenvc_dit.h) at
their borders, on the CPU: calls in place, and sizes at and beyond what a call
can do.  Every call here is refused before any HIP call, so the fake addresses are
never dereferenced."""
import ctypes

import pytest

from paper_2607_28144_amd import _lib

A, B, C, D, E = (0x10000000 + (i << 33) for i in range(5))  # 256-byte aligned, far apart
LN, NONE = _lib.Norm(1, 1e-6, None, None), _lib.Norm(0, 1e-6, None, None)
BF16, F32 = _lib.BF16, _lib.F32
INV, UNS = _lib.ERR_INVALID_ARG, _lib.ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def refused(lib, status, word, st):
    assert st == status, (st, lib.regenvc_last_error())
    assert word in lib.regenvc_last_error().decode(), lib.regenvc_last_error()


def forward(lib, **kw):
    a = dict(dict(x=A, ldx=64, y=B, ldy=64, t=F32, gate=None, xo=A, ldxo=64, h=C, ldh=64, rows=10, C=64), **kw)
    v = _lib.RowVectors(a["gate"], None, None, 64, 0)
    return lib.regenvc_residual_norm_fwd(a["x"], a["ldx"], a["y"], a["ldy"], a["t"], NONE, LN, v, 1.0, a["xo"], a["ldxo"],
                                         a["h"], a["ldh"], a["rows"], a["C"], None)


@pytest.mark.parametrize("t", [BF16, F32])
def test_forward_in_place_exempts_the_stream_alone(lib, t):
    """x_out over x; at that address lies nothing else, in any row stride."""
    for ld in (64, 72):
        refused(lib, INV, "x_out overlaps h", forward(lib, t=t, h=A, ldh=ld))
        refused(lib, INV, "x_out overlaps y", forward(lib, t=t, y=A, ldy=ld))
    refused(lib, INV, "x_out overlaps gate", forward(lib, t=t, gate=A))
    refused(lib, INV, "x_out overlaps h", forward(lib, t=t, h=A + 256))
    refused(lib, INV, "x_out overlaps x", forward(lib, t=t, ldxo=72))
    # in place alone is let through: it is a later pair that speaks
    refused(lib, INV, "h overlaps y", forward(lib, t=t, h=B))


def backward(lib, **kw):
    a = dict(dict(x=A, y=B, gh=C, ldgh=64, gx=D, ldgx=64, dx=D, lddx=64, dy=E, lddy=64, t=F32, dgate=None, rows=10), **kw)
    v = _lib.RowVectors(E + (1 << 32), None, None, 64, 0)
    return lib.regenvc_residual_norm_bwd(a["x"], 64, a["y"], 64, a["t"], NONE, LN, v, 1.0, a["gh"], a["ldgh"], a["gx"],
                                         a["ldgx"], a["dx"], a["lddx"], a["dy"], a["lddy"], _lib.NormGrads(dgate=a["dgate"]),
                                         a["rows"], 64, None, 0, None)


@pytest.mark.parametrize("t", [BF16, F32])
def test_backward_in_place_exempts_the_stream_gradient_alone(lib, t):
    """dx over gx; at that address lies nothing else."""
    for ld in (64, 72):
        refused(lib, INV, "dx overlaps dy", backward(lib, t=t, dy=D, lddy=ld))
        refused(lib, INV, "dx overlaps gh", backward(lib, t=t, gh=D, ldgh=ld))
    refused(lib, INV, "dx overlaps dgate", backward(lib, t=t, dgate=D))
    refused(lib, INV, "dx overlaps x_out", backward(lib, t=t, x=D))
    refused(lib, INV, "dx overlaps y", backward(lib, t=t, y=D))
    refused(lib, INV, "dx overlaps gx", backward(lib, t=t, lddx=72))
    refused(lib, INV, "dy overlaps gh", backward(lib, t=t, dy=C))


def workspace(lib, rows, C=64, group_rows=0, sums=(3, 2), n_cu=256):
    n = ctypes.c_int64(-7)
    return lib.regenvc_residual_norm_bwd_workspace(rows, C, group_rows, *sums, n_cu, ctypes.byref(n)), n.value


@pytest.mark.parametrize("C,limit", [(64, 1 << 26), (2048, 1 << 26), (2056, 1 << 24), (8192, 1 << 24)])
def test_workspace_query_refuses_the_rows_that_the_call_refuses(lib, C, limit):
    """... and gives no size for them; sums of sizes that pass 32 bits neither end the process nor come out as 0."""
    for rows in (limit, (1 << 30) + 8, 1500000000, (1 << 31) - 1):
        for group_rows in (0, 1, rows - 1, (1 << 31) - 1):
            st, n = workspace(lib, rows, C, group_rows)
            refused(lib, UNS, "must be below", st)
            assert n == -7


def test_workspace_query_for_any_number_of_compute_units(lib):
    """At least a row of C for each sum over all rows, and no more than one for every sum and row: a group has at most
    group_rows segments, so there are at most ceil(rows / group_rows) group_rows < rows + group_rows of them (the last
    group's may be empty)."""
    for rows, C, group_rows in ((10920, 1536, 1560), (100, 64, 0), (5000, 8192, 7), (1 << 20, 64, 1)):
        for n_cu in (1, 304, 1 << 20, 2000000000, (1 << 31) - 1):
            st, n = workspace(lib, rows, C, group_rows, n_cu=n_cu)
            assert st == _lib.OK and 2 * C * 4 <= n < 5 * (rows + group_rows + 1) * C * 4, (rows, C, group_rows, n_cu, n)


@pytest.mark.parametrize("C,most", [(8, (1 << 26) - 4), (2048, (1 << 26) - 4), (2056, (1 << 24) - 1), (8192, (1 << 24) - 1)])
def test_most_rows_are_those_of_one_launch(lib, C, most):
    """A launch has less than 2^32 threads: four rows to a workgroup of 256, or one beyond 2048 channels."""
    per = 4 if C <= 2048 else 1
    assert -(-most // per) * 256 < 1 << 32 <= -(-(most + 1) // per) * 256
    ld = dict(ldx=C, ldxo=C, ldy=C, ldh=C, C=C, xo=None)
    refused(lib, INV, "a NULL data pointer", forward(lib, rows=most, **ld))  # the sizes are in order
    refused(lib, UNS, "must be below", forward(lib, rows=most + 1, **ld))
    assert workspace(lib, most, C)[0] == _lib.OK
    refused(lib, UNS, "must be below", workspace(lib, most + 1, C)[0])
