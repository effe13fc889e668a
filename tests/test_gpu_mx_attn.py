"""GPU parity of the MXFP4 key/value cache (append, values, attention) against
the fp64 oracle (oracle/mx.py).

Bounds.  The cache's values are exact.  A score q.k is a sum of D exact
products in fp32: off by at most 12 * 2^-24 sum |q||k| (D / 32 additions of
32-deep sums, each within 2 roundings, and one more for D = 64's order), times
scale; the exponent's argument is rounded once more, relative to its size.
Call that es, the largest over a row's keys.  Weights are rounded to bf16 (half
a step, 2^-8) and O is divided by the sum of the rounded weights, so
|dO| <= (2^-8 + 2 es)(sum p|v| + |O|), plus the output's own rounding; LSE takes
unrounded weights: es, and the roundings of a sum of n terms in lanes of n / 8.
"""
import math

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


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def filled(B, cap, heads, D, seed, sharp=1.0):
    """A cache full of tokens, and the values that it holds [B, cap, heads, D]."""
    rng = np.random.default_rng(seed)
    k, v = synth.normal_bf16(rng, (B, cap, heads, D), sharp), synth.normal_bf16(rng, (B, cap, heads, D))
    c = mx().KvCache(B, cap, heads, D)
    c.append(bf16(k), bf16(v))
    return c, omx.values(odit.widen(k)), omx.values(odit.widen(v))


def check(name, o, lse, q, k, v, lens, scale, bf16_out=True):
    ro, rl, mag = omx.attn(q, k, v, lens, scale)
    B, S, H, D = q.shape
    G = H // k.shape[2]
    es = np.zeros((B, S, H, 1))
    for b in range(B):
        n = int(lens[b])
        if n == 0:
            continue
        for h in range(H):
            a = np.abs(q[b, :, h]) @ np.abs(k[b, :n, h // G]).T * scale
            es[b, :, h, 0] = a.max(1) * (12 * 2.0 ** -24 + 2 * 2.0 ** -24) + 2.0 ** -22
    tol = (2.0 ** -8 + 2 * es) * (mag + np.abs(ro)) + (2.0 ** -8 if bf16_out else 2.0 ** -22) * np.abs(ro) + 1e-30
    go, gl = host(o), host(lse)
    err = np.abs(go - ro)
    n = max(1, int(max(lens)))
    tl = es[..., 0].transpose(0, 2, 1) + (n / 8 + 64) * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(np.isfinite(rl), rl, 0))
    empty = np.isneginf(rl)
    el = np.where(empty, np.where(np.isneginf(gl), 0.0, np.inf), np.abs(np.where(empty, 0, gl) - np.where(empty, 0, rl)))
    print(f"[mx attn] {name}: max|dO|={err.max():.3e} ({(err / tol).max():.3f} of the bound) max|dLSE|={el.max():.3e} "
          f"({(el / tl).max():.3f})", flush=True)
    assert np.isfinite(go).all() and (err <= tol).all() and (el <= tl).all()


# rows for a key head from 1 to many (each kernel and its borders), lengths around tiles and ranges
CASES = [(1, 1, 1, 1, 64, 40, [1]), (1, 1, 2, 2, 128, 300, [300]), (2, 1, 12, 12, 128, 1000, [1000, 31]),
         (3, 1, 16, 2, 64, 700, [0, 33, 700]), (2, 16, 4, 4, 128, 513, [512, 64]), (1, 17, 3, 3, 64, 2048, [1999]),
         (2, 5, 12, 4, 128, 260, [255, 257]), (1, 33, 2, 1, 128, 600, [577]), (1, 64, 3, 3, 128, 1100, [1100]),
         (1, 65, 2, 2, 64, 320, [65]), (2, 130, 4, 2, 128, 2500, [2431, 0]), (1, 300, 3, 3, 64, 4000, [3777]),
         (1, 129, 5, 1, 128, 200, [63]), (1, 1560, 2, 2, 128, 1600, [1560])]


@pytest.mark.parametrize("B,S,H,heads,D,cap,lens", CASES)
@pytest.mark.parametrize("f32", [False, True])
def test_attention(B, S, H, heads, D, cap, lens, f32):
    c, k, v = filled(B, cap, heads, D, B * 1000 + S)
    q = synth.normal_bf16(np.random.default_rng(S), (B, S, H, D))
    scale = synth.default_scale(D)
    o, lse = mx().attn_cache_fwd(bf16(q), c, ints(lens), out_dtype=torch.float32 if f32 else torch.bfloat16)
    check(f"{(B, S, H, heads, D, cap, lens)}", o, lse, odit.widen(q), k, v, lens, scale, not f32)


@pytest.mark.parametrize("S,cap,ranges", [(200, 1024, 2), (200, 1600, 3), (1, 1030, 4), (2, 1300, 5), (20, 1800, 7), (1, 2100, 8),
                                          (3, 2400, 9), (30, 5130, 20), (1, 16500, 64)])
def test_joined_ranges(S, cap, ranges):
    """Every form of the joining of key ranges, all of them in use and most of them empty."""
    import ctypes
    from paper_2607_28144_amd import _lib
    B, H, D = 2, 1, 64
    p = _lib.MxAttnPlan()
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    assert _lib.load().regenvc_mx_attn_cache_plan_query(B, H, H, S, cap, D, n_cu, ctypes.byref(p)) == 0
    assert p.key_ranges == ranges
    c, k, v = filled(B, cap, H, D, cap)
    q = synth.normal_bf16(np.random.default_rng(S), (B, S, H, D))
    for lens in ([cap, 70], [cap - 1, 0], [129, cap // 2]):
        o, lse = mx().attn_cache_fwd(bf16(q), c, ints(lens), out_dtype=torch.float32)
        check(f"S={S} cap={cap} {lens}", o, lse, odit.widen(q), k, v, lens, synth.default_scale(D), False)


@pytest.mark.parametrize("S", [1, 40, 200])
def test_sharp_scores_and_scales(S):
    """Scores of both signs far apart, a scale of 0 (all places alike) and one of 1."""
    B, H, D, cap = 1, 3, 128, 777
    c, k, v = filled(B, cap, H, D, 3, sharp=8.0)
    q = synth.normal_bf16(np.random.default_rng(S), (B, S, H, D), 4.0)
    for scale in (0.0, synth.default_scale(D), 1.0):
        o, lse = mx().attn_cache_fwd(bf16(q), c, ints([cap]), scale=scale, out_dtype=torch.float32)
        check(f"sharp S={S} scale={scale:.3f}", o, lse, odit.widen(q), k, v, [cap], scale, False)


@pytest.mark.parametrize("S", [1, 20, 50, 200])
def test_what_lies_behind_the_length_is_not_read(S):
    """NaN blocks behind a length (in its last tile, and whole tiles) change nothing; within it they do."""
    B, H, D, cap = 2, 2, 128, 400
    c, k, v = filled(B, cap, H, D, 4)
    q = bf16(synth.normal_bf16(np.random.default_rng(1), (B, S, H, D)))
    lens = ints([101, 256])
    o, lse = mx().attn_cache_fwd(q, c, lens)
    for t in (c.k_scales, c.v_scales):
        t[0, :, 101:] = 255
        t[1, :, 256:] = 255
    o2, lse2 = mx().attn_cache_fwd(q, c, lens)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    c.k_scales[0, 1, 50] = 255
    c.v_scales[1, 0, 200, 2] = 255
    o3, lse3 = mx().attn_cache_fwd(q, c, lens)
    assert bool(torch.isnan(o3[0, :, 1]).all()) and bool(torch.isnan(lse3[0, 1]).all())
    assert torch.equal(o3[0, :, 0], o[0, :, 0]) and torch.equal(o3[1, :, 1], o[1, :, 1])
    assert bool(torch.isnan(o3[1, :, 0, 64:96]).all()) and torch.equal(o3[1, :, 0, :64], o[1, :, 0, :64])


@pytest.mark.parametrize("D,heads,cap", [(64, 3, 7), (128, 2, 50)])
def test_append_places_and_values(D, heads, cap):
    """Starts, counts and wrapping; more tokens than the cache holds; a negative start and counts of none: every
    place holds what the rule says, the others what they held."""
    rng = np.random.default_rng(cap)
    B, S = 6, cap + 5
    c = mx().KvCache(B, cap, heads, D)
    k0, v0 = synth.normal_bf16(rng, (B, cap, heads, D)), synth.normal_bf16(rng, (B, cap, heads, D))
    c.append(bf16(k0), bf16(v0))
    wide = synth.normal_bf16(rng, (B, S, 2, heads, D))
    t = bf16(wide)
    start = [0, cap - 2, 3 * cap + 1, -1, 2, 5]
    count = [S, 4, cap, 5, 0, -3]
    c.append(t[:, :, 0], t[:, :, 1], ints(start), ints(count))
    ref = [odit.widen(k0), odit.widen(v0)]
    for b in range(B):
        n = max(0, min(count[b], S))
        for i in range(max(0, n - cap), n):
            if start[b] >= 0:
                for j in range(2):
                    ref[j][b, (start[b] + i) % cap] = odit.widen(wide[b, i, j])
    for dt in (torch.float32, torch.bfloat16):
        k, v = c.values(dt)
        assert np.array_equal(host(k), omx.values(ref[0])) and np.array_equal(host(v), omx.values(ref[1]))


def test_append_nonfinite_and_defaults():
    c = mx().KvCache(1, 8, 1, 64)
    k = torch.randn(1, 3, 1, 64, device="cuda").bfloat16()
    v = k.clone()
    k[0, 1, 0, 40] = float("inf")
    c.append(k, v)
    kk, vv = c.values()
    assert bool(torch.isnan(kk[0, 1, 0, 32:]).all()) and bool(torch.isfinite(kk[0, 1, 0, :32]).all())
    assert bool((kk[0, 3:] == 0).all()) and bool(torch.isfinite(vv).all())
    c.append(k[:, :0], v[:, :0])


def test_layouts_of_q_and_o():
    """Head-major q, o as a slice of a larger tensor, and what lies around it as it was."""
    B, S, H, D, cap = 2, 20, 4, 128, 300
    c, _, _ = filled(B, cap, 2, D, 8)
    q = bf16(synth.normal_bf16(np.random.default_rng(2), (B, H, S, D))).transpose(1, 2)
    lens = ints([300, 17])
    ref, lse = mx().attn_cache_fwd(q.contiguous(), c, lens)
    big = torch.full((B, S + 2, H, D + 16), 5.0, dtype=torch.bfloat16, device="cuda")
    o, _ = mx().attn_cache_fwd(q, c, lens, out=big[:, 1:-1, :, 8:8 + D], return_lse=False)
    assert torch.equal(o, ref)
    big[:, 1:-1, :, 8:8 + D] = 5.0
    assert bool((big == 5.0).all())


def test_lens_held_and_max_len():
    """Lengths beyond the capacity and below 0; a plan for shorter sequences than there are."""
    B, S, H, D, cap = 3, 4, 2, 64, 900
    c, _, _ = filled(B, cap, H, D, 9)
    q = bf16(synth.normal_bf16(np.random.default_rng(2), (B, S, H, D)))
    a = mx().attn_cache_fwd(q, c, ints([cap, 0, 500]), out_dtype=torch.float32)
    b = mx().attn_cache_fwd(q, c, ints([cap + 77, -5, 500]), out_dtype=torch.float32)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    s = mx().attn_cache_fwd(q, c, ints([cap, 0, 500]), max_len=10, out_dtype=torch.float32)
    assert float((s[0] - a[0]).abs().max()) < 2.0 ** -6 and float((s[1] - a[1])[[0, 2]].abs().max()) < 1e-4
    assert bool((a[0][1] == 0).all()) and bool(torch.isneginf(a[1][1]).all())
    n = mx().attn_cache_fwd(q, c, None, max_len=500, out_dtype=torch.float32)
    f = mx().attn_cache_fwd(q, c, ints([500, 500, 500]), max_len=500, out_dtype=torch.float32)
    assert torch.equal(n[0], f[0])


@pytest.mark.parametrize("S", [1, 30, 300])
def test_captured_with_growing_lengths(S):
    """One graph of append and attention, replayed as the sequence grows (lengths and starts live on the device)."""
    B, H, D, cap = 1, 3, 128, 1024
    c = mx().KvCache(B, cap, H, D)
    eager = mx().KvCache(B, cap, H, D)
    rng = np.random.default_rng(S)
    q = bf16(synth.normal_bf16(rng, (B, S, H, D)))
    k, v = (torch.empty(B, S, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    start, lens = ints([0]), ints([0])

    def step(cache):
        cache.append(k, v, start)
        return mx().attn_cache_fwd(q, cache, lens)
    step(c)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o, lse = step(c)
    for t in range(4):
        k.copy_(bf16(synth.normal_bf16(rng, (B, S, H, D))))
        v.copy_(bf16(synth.normal_bf16(rng, (B, S, H, D))))
        start.fill_(t * S)
        lens.fill_(min(cap, (t + 1) * S))
        g.replay()
        eo, el = step(eager)
        torch.cuda.synchronize()
        assert torch.equal(o, eo) and torch.equal(lse, el)


def test_joined_with_fresh_tokens():
    """Attention over the cache merged with attention over a chunk that is still in bf16 (partials and LSE merge):
    what attention over both together gives."""
    from paper_2607_28144_amd import api
    B, S, H, D, cap = 1, 260, 3, 128, 640
    c, k, v = filled(B, cap, H, D, 12)
    rng = np.random.default_rng(3)
    q, kn, vn = (synth.normal_bf16(rng, (B, S, H, D)) for _ in range(3))
    scale = synth.default_scale(D)
    o1, l1 = mx().attn_cache_fwd(bf16(q), c, ints([600]), out_dtype=torch.float32)
    o2, l2 = api.attn_partial_fwd(bf16(q), bf16(kn), bf16(vn))
    o, lse = api.lse_merge([o1, o2], [l1, l2])
    kk, vv = np.concatenate([k[:, :600], odit.widen(kn)], 1), np.concatenate([v[:, :600], odit.widen(vn)], 1)
    check("joined", o, lse, odit.widen(q), kk, vv, [600 + S], scale)
