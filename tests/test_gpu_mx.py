"""GPU parity of the MXFP4 kernels (include/regenvc_mx.h) against the fp64
oracle (oracle/mx.py): quantisation bit for bit, linear layers within the
bound of their fp32 sums.

A linear layer's products are exact in fp32 (two-bit magnitudes under powers of
two), so its error is that of adding K of them: at most one rounding per
addition of a 128-deep partial sum, which itself is taken to be off by no more
than 4 roundings, all relative to the sum of magnitudes:
(2 * steps + 8 + joins of waves) * 2^-24 * sum |a||w|.  A bf16 output adds half a
step, 2^-8 of the value; GELU has a slope of at most 1.13 and an exponential
good to 1e-6.
"""
import numpy as np
import pytest

from oracle import dit as odit
from oracle import mx as omx
from paper_2607_28144_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def mx():
    from paper_2607_28144_amd import mx as m
    return m


def bf16(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).cuda()


def host(t):
    return t.double().cpu().numpy()


def same(got, ref):
    """Equal value by value, NaN where NaN."""
    return np.array_equal(got, ref, equal_nan=True)


def edge_rows(K):
    """Rows that hold every rounding case: ties, saturation, zeros, tiny and huge blocks, blocks with infinities."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((24, K)).astype(np.float32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 7.9, 4.0, 0.2500001, 5.0000005], dtype=np.float32)
    for r, s in enumerate((1.0, -1.0, 2.0 ** 40, 2.0 ** -60, -2.0 ** 120)):
        n = min(K, len(ties))
        x[r, :n] = ties[-n:] * np.float32(s)
        x[r, n:32] = 0.0
    x[5] = 0.0
    x[6, :32] = -0.0
    x[7] *= np.float32(2.0 ** -130)            # subnormal inputs
    x[8, 3] = np.inf
    x[9, 40 % K] = np.nan
    x[10, K - 1] = -np.inf
    x[11] *= np.float32(1e38)
    x[12, :32] = np.float32(2.0 ** -126)
    x[13, :32] = np.float32(3.3e38)
    x[14, 0], x[14, 1:32] = np.float32(1e30), np.float32(1e-30)
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [8, 32, 72, 256, 264, 512, 1536, 1544])
def test_quantize_is_the_definition(K, dtype):
    x = torch.from_numpy(edge_rows(K))
    x = (x.to(torch.bfloat16) if dtype == "bf16" else x).cuda()
    m = mx().quantize(x)
    ref = omx.values(host(x))
    assert same(host(mx().dequantize(m)), ref)
    b = mx().dequantize(m, torch.bfloat16)
    assert same(host(b), host(torch.from_numpy(ref).to(torch.float32).to(torch.bfloat16)))


@pytest.mark.parametrize("rows", [1, 15, 16, 17, 100])
def test_quantize_strided_and_layout(rows):
    """A view with a row stride; the codes and scales lie as regenvc_mx.h says, filled up with zeros."""
    K = 328
    rng = np.random.default_rng(rows)
    wide = torch.from_numpy(rng.standard_normal((rows, 400)).astype(np.float32)).to(torch.bfloat16).cuda()
    x = wide[:, 8:8 + K]
    m = mx().quantize(x)
    code, byte = omx.encode(host(x))
    got = m.codes.cpu().numpy().reshape(rows, -1)
    got = np.stack([got & 15, got >> 4], -1).reshape(rows, -1)
    ref = np.zeros((rows, 512), dtype=int)
    ref[:, : code.shape[1] * 32] = code.reshape(rows, -1)
    assert np.array_equal(got, ref)
    sc = m.scales.cpu().numpy().reshape(-1, 2, 4, 16, 2)  # [16 rows][step][g][row][block of the pair]
    sc = sc.transpose(0, 3, 1, 2, 4).reshape(-1, 16)
    ref = np.zeros((-(-rows // 16) * 16, 16), dtype=int)
    ref[:rows, : byte.shape[1]] = byte
    assert np.array_equal(sc, ref)


def linear_case(M, N, K, seed):
    rng = np.random.default_rng(seed)
    a = synth.normal_bf16(rng, (M, K))
    a = synth.f32_to_bf16_bits(synth.bf16_bits_to_f32(a) * np.exp(0.7 * rng.standard_normal(K)).astype(np.float32))
    return a, synth.normal_bf16(rng, (N, K), 0.02), synth.normal_bf16(rng, (N,), 0.02)


def check(name, got, ref, tol):
    err = np.abs(got - ref)
    ratio = float((err / tol).max()) if err.size else 0.0
    print(f"[mx] {name}: max|d|={err.max() if err.size else 0:.3e} err/bound={ratio:.3f}", flush=True)
    assert np.isfinite(got).all() and ratio <= 1.0, f"{name}: err/bound {ratio}"


# every kernel and its borders: one to 64 rows (few-row kernels, K in few and in many steps), tiles of
# each shape, ragged rows and channels, K that ends inside a block, a half step and a step
SHAPES = [(1, 16, 8), (1, 1536, 1536), (3, 48, 40), (16, 272, 264), (17, 272, 2312), (33, 1536, 1536), (64, 160, 8960),
          (65, 16, 8), (65, 144, 72), (130, 272, 256), (129, 400, 512), (300, 1552, 1544), (577, 1536, 768),
          (1365, 1536, 8960), (700, 8960, 1536), (2500, 1040, 1000), (5, 4624, 1544), (16, 1536, 2056)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("given", ["bf16", "mx"])
def test_linear(M, N, K, given):
    a, w, b = linear_case(M, N, K, M + N + K)
    A, W, Bv = omx.values(odit.widen(a)), omx.values(odit.widen(w)), odit.widen(b)
    y = A @ W.T + Bv
    steps = -(-K // 256)
    slack = (2 * steps + 16) * 2.0 ** -24 * (np.abs(A) @ np.abs(W).T + np.abs(Bv))
    da, dw, db = bf16(a), mx().quantize(bf16(w)), bf16(b)
    if given == "mx":
        da = mx().quantize(da)
    rng = np.random.default_rng(1)
    gate, x0 = rng.standard_normal(N).astype(np.float32), rng.standard_normal((M, N)).astype(np.float32)
    out = mx().linear_fwd(da, dw, db)
    out_g = mx().linear_fwd(da, dw, db, epilogue="bias_gelu")
    x = torch.from_numpy(x0).cuda()
    mx().linear_fwd(da, dw, db, epilogue="gated_residual", gate=torch.from_numpy(gate).cuda(), out=x)
    nb = mx().linear_fwd(da, dw)
    torch.cuda.synchronize()
    name = f"{M}x{N}x{K} {given}"
    check(name + " bias", host(out), y, 2.0 ** -8 * np.abs(y) + slack + 1e-30)
    check(name + " none", host(nb), y - Bv, 2.0 ** -8 * np.abs(y - Bv) + slack + 1e-30)
    g = odit.gelu_tanh(y)
    check(name + " gelu", host(out_g), g, 2.0 ** -8 * np.abs(g) + 1.13 * slack + 1e-6)
    ref = x0 + gate.astype(np.float64) * y
    check(name + " gated", host(x), ref, np.abs(gate) * slack + 2.0 ** -22 * (np.abs(x0) + np.abs(gate * y)) + 1e-30)


def test_linear_strides_and_surroundings():
    """Strided a and out; what lies around the output stays as it was."""
    for M in (5, 40, 200):
        N, K = 272, 328
        a, w, b = linear_case(M, N, K, M)
        wide = torch.full((M, K + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, 8:8 + K] = bf16(a)
        dw = mx().quantize(bf16(w))
        big = torch.full((M + 2, N + 48), 7.0, dtype=torch.bfloat16, device="cuda")
        mx().linear_fwd(wide[:, 8:8 + K], dw, bf16(b), out=big[1:-1, 16:16 + N])
        ref = mx().linear_fwd(bf16(a), dw, bf16(b))
        assert torch.equal(big[1:-1, 16:16 + N], ref)
        big[1:-1, 16:16 + N] = 7.0
        assert bool((big == 7.0).all())


@pytest.mark.parametrize("M", [2, 40, 300])
def test_linear_nonfinite_rows(M):
    """A NaN or an infinity in a row of a reaches that row only, whole; a channel of W likewise."""
    N, K = 272, 1544
    a, w, b = linear_case(M, N, K, 9)
    da, wt = bf16(a), bf16(w)
    clean = mx().linear_fwd(da, mx().quantize(wt), bf16(b))
    da[1, 700] = float("inf")
    wt[33, 5] = float("nan")
    got = mx().linear_fwd(da, mx().quantize(wt), bf16(b))
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[1] = True
    bad[:, 33] = True
    assert bool(torch.isnan(got[bad]).all())
    assert torch.equal(got[~bad], clean[~bad])


def test_linear_empty():
    """No rows, no channels: nothing; no columns: the epilogue of 0."""
    def some(*shape):
        return torch.randn(*shape, device="cuda").bfloat16()
    w = mx().quantize(some(32, 64))
    assert mx().linear_fwd(some(0, 64), w).shape == (0, 32)
    assert mx().linear_fwd(some(4, 64), mx().quantize(some(0, 64))).shape == (4, 0)
    assert mx().dequantize(mx().quantize(some(0, 64))).shape == (0, 64)
    bias = some(48)
    for M in (3, 40, 200):
        for a in (some(M, 0), mx().quantize(some(M, 0))):
            assert torch.equal(mx().linear_fwd(a, mx().quantize(some(48, 0)), bias), bias.expand(M, 48))
    x = torch.randn(200, 48, device="cuda")
    ref = x + bias.float()
    mx().linear_fwd(some(200, 0), mx().quantize(some(48, 0)), bias, epilogue="gated_residual", out=x)
    assert torch.equal(x, ref)


@pytest.mark.parametrize("M,N,K", [(7, 272, 1536), (40, 272, 1536), (300, 1536, 8960)])
def test_linear_captured_and_streams(M, N, K):
    """Captured into a graph and replayed between eager calls on another stream: each as the first eager call."""
    a, w, b = linear_case(M, N, K, 3)
    da, dw, db = bf16(a), mx().quantize(bf16(w)), bf16(b)
    ref = mx().linear_fwd(da, dw, db).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mx().linear_fwd(da, dw, db)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = mx().linear_fwd(da, dw, db)
    for _ in range(3):
        out.zero_()
        g.replay()
        with torch.cuda.stream(side):
            other = mx().linear_fwd(da, dw, db)
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(other, ref)
