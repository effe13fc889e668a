"""MXFP4 linear layers, each kind of tile where workgroups walk several tiles and
where they have one: the copies aimed at the next tile, its biases, and an
output stored beside copies under way.  Against products in 64 bits of the
operands' values, which are exact.

The bound is that of fp32 sums: products are exact, at most one rounding per
addition of a 128-deep partial sum and four within it, relative to the sum of
magnitudes, (2 steps + 16) 2^-24 sum |a||w|; half a step of bf16, 2^-8 of the
value; GELU has a slope of at most 1.13 and an exponential good to 1e-6; the
gated residual's product and sum are two more fp32 roundings.
"""
import ctypes

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


# (rows, columns of the tile, workgroups per compute unit): by epilogue, sizes with ragged rows, channels and K
CASES = [
    ("bias", 128, 128, 2, True, (2570, 3216, 776)), ("bias_gelu", 128, 128, 2, True, (2570, 3216, 776)),
    ("gated_residual", 128, 128, 2, True, (5496, 1872, 776)), ("bias_gelu", 128, 128, 2, True, (1419, 9040, 1544)),
    ("bias", 64, 128, 2, True, (1424, 5552, 776)), ("bias_gelu", 64, 128, 2, True, (1419, 5392, 272)),
    ("gated_residual", 64, 128, 2, True, (1281, 3904, 264)), ("bias", 64, 128, 2, False, (68, 8336, 296)),
    ("bias_gelu", 64, 128, 2, False, (67, 8528, 816)), ("gated_residual", 64, 128, 2, False, (130, 6208, 304)),
    ("bias", 96, 96, 1, True, (5975, 656, 5032)), ("bias_gelu", 96, 96, 1, True, (1286, 3152, 1288)),
    ("gated_residual", 96, 96, 1, True, (475, 8384, 264)), ("gated_residual", 96, 96, 1, True, (4746, 848, 3664)),
    ("bias", 64, 64, 2, True, (5527, 656, 1840)), ("bias_gelu", 64, 64, 2, True, (300, 7824, 280)),
    ("gated_residual", 64, 64, 2, True, (201, 8480, 280)),
    # 128 x 128 with four stages, one workgroup per compute unit
    ("bias", 128, 128, 1, False, (205, 8416, 1576)), ("bias_gelu", 128, 128, 1, False, (199, 8256, 1504)),
    ("gated_residual", 128, 128, 1, False, (454, 6176, 1352)), ("bias", 128, 128, 1, True, (1423, 3312, 8880)),
    ("bias_gelu", 128, 128, 1, True, (1423, 3312, 8880)),
]


def near(name, got, ref, tol):
    ratio = float(((got.double() - ref).abs() / tol).max())
    print(f"[mx tiles] {name}: {ratio:.3f} of the bound", flush=True)
    assert ratio <= 1.0, name


@pytest.mark.parametrize("epilogue,bm,bn,per_cu,several,size", CASES)
def test_tiles(epilogue, bm, bn, per_cu, several, size):
    from paper_2607_28144_amd import _lib, dit, mx
    M, N, K = size
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    p = _lib.TilePlan()
    assert _lib.load().regenvc_mx_linear_plan_query(M, N, K, dit.EPI[epilogue], n_cu, ctypes.byref(p)) == 0
    assert (p.rows, p.cols) == (bm, bn) and (-(-M // bm) * -(-N // bn) > per_cu * n_cu) == several
    g = torch.Generator(device="cuda")
    g.manual_seed(M + N + K)

    def r(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std
    a = (r(M, K) * torch.exp(0.7 * r(K))).bfloat16()
    w, b, gate = mx.quantize(r(N, K, std=0.02).bfloat16()), r(N, std=0.02).bfloat16(), r(N)
    A, W = mx.dequantize(mx.quantize(a)).double(), mx.dequantize(w).double()
    y = torch.mm(A, W.t()) + b.double()
    slack = (2 * -(-K // 256) + 16) * 2.0 ** -24 * (torch.mm(A.abs(), W.abs().t()) + b.double().abs())
    # the output within a larger tensor, whose rest stays as it was
    gated = epilogue == "gated_residual"
    big = torch.full((M + 2, N + 48), 7.0, dtype=torch.float32 if gated else torch.bfloat16, device="cuda")
    out = big[1:-1, 16:16 + N]
    x = r(M, N)
    if gated:
        out.copy_(x)
    mx.linear_fwd(a, w, b, epilogue=epilogue, gate=gate if gated else None, out=out)
    name = f"{M} x {N} x {K} {epilogue}"
    if gated:
        gy = gate.double() * y
        near(name, out, x.double() + gy, gate.double().abs() * slack + 2.0 ** -22 * (x.double().abs() + gy.abs()) + 1e-30)
    else:
        ref = y
        if epilogue == "bias_gelu":
            ref = 0.5 * y * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (y + 0.044715 * y ** 3)))
            slack = 1.13 * slack + 1e-6
        near(name, out, ref, 2.0 ** -8 * ref.abs() + slack + 1e-30)
    out.fill_(7.0)
    assert bool((big == 7.0).all())
