"""Sizes at and beyond what the calls of include/regenvc_mx.h can do, on the CPU:
refused before any HIP call, so the fake addresses are never dereferenced."""
import ctypes

import pytest

from paper_2607_28144_amd import _lib

A, B, C = (0x10000000 + (i << 40) for i in range(3))
INV, UNS = _lib.ERR_INVALID_ARG, _lib.ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def refused(lib, status, word, st):
    assert st == status, (st, lib.regenvc_last_error())
    assert word in lib.regenvc_last_error().decode(), lib.regenvc_last_error()


def test_most_rows_of_a_dequantisation_are_those_of_one_launch(lib):
    """A launch has less than 2^32 threads: four rows to a workgroup of 256.  The conversion to MXFP4, with sixteen,
    takes every matrix that there are sizes for."""
    most = (1 << 26) - 4
    assert -(-most // 4) * 256 < 1 << 32 <= -(-(most + 1) // 4) * 256
    d = lib.regenvc_mx_dequantize
    refused(lib, INV, "a NULL data pointer", d(A, B, None, _lib.F32, 8, most, 8, None))
    refused(lib, UNS, "rows, at most", d(A, B, C, _lib.F32, 8, most + 1, 8, None))
    n, m = ctypes.c_int64(), ctypes.c_int64()
    assert lib.regenvc_mx_bytes((1 << 26) - 1, 8, ctypes.byref(n), ctypes.byref(m)) == _lib.OK
    refused(lib, INV, "a NULL data pointer", lib.regenvc_mx_quantize(None, _lib.BF16, 8, A, B, (1 << 26) - 1, 8, None))


def test_linear_workspace_holds_the_activations():
    """What a bf16 operand needs is never less than its codes and scales, but for the rows that the few-row kernel
    brings to MXFP4 itself."""
    pytest.importorskip("torch")
    from paper_2607_28144_amd import mx
    for M, N, K in [(17, 16, 8), (65, 16, 8), (1365, 1536, 8960), (10920, 8960, 1536), (200, 8960, 8960), (16, 1536, 2056)]:
        assert mx.linear_workspace_bytes(M, N, K, False) >= sum(mx.mx_bytes(M, K))
        assert mx.linear_workspace_bytes(M, N, K, True) == 0
    assert mx.linear_workspace_bytes(16, 1536, 2048, False) == 0
