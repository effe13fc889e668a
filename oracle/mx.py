"""Reference oracle of MXFP4 and of attention over a cache held in it -- TEST
INFRASTRUCTURE ONLY: plain float64 numpy definitions, nothing shared with the
product.

A block of 32 values has one scale 2^e, e = max(-127, floor(log2 max|x|) - 2),
and codes of four bits: a sign and the index of a magnitude in GRID, the one
nearest to |x| / 2^e, ties to the even index, the largest for all beyond it.  A
block with an infinity or NaN has scale byte 255 and stands for NaN.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def encode(x: np.ndarray):
    """Codes (0..15, sign in bit 3) and scale bytes of x [..., n], the last
    block filled up with zeros: [..., blocks, 32] and [..., blocks]."""
    x = np.asarray(x, dtype=np.float64)
    n = x.shape[-1]
    x = np.concatenate([x, np.zeros(x.shape[:-1] + (-n % 32,))], -1).reshape(x.shape[:-1] + (-1, 32))
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    top = np.abs(x).max(-1)
    e = np.maximum(np.frexp(top)[1] - 1 - 2, -127)  # frexp: top = m 2^k with m in [0.5, 1)
    e = np.where(top == 0, -127, e)
    m = np.abs(x) / np.ldexp(1.0, e)[..., None]
    dist = np.abs(m[..., None] - GRID)  # exact: m has few bits
    near = dist.min(-1, keepdims=True)
    tied = dist == near
    even = tied & (np.arange(8) % 2 == 0)
    idx = np.where(tied.sum(-1) > 1, even.argmax(-1), tied.argmax(-1))
    code = idx + 8 * np.signbit(x)
    return np.where(bad[..., None], 0, code), np.where(bad, 255, e + 127)


def decode(code: np.ndarray, byte: np.ndarray, n: int) -> np.ndarray:
    """The values [..., n] of codes [..., blocks, 32] and scale bytes [..., blocks]."""
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0) * np.ldexp(1.0, byte - 127)[..., None]
    v = np.where((byte == 255)[..., None], np.nan, v)
    return v.reshape(v.shape[:-2] + (-1,))[..., :n]


def values(x: np.ndarray) -> np.ndarray:
    """x [..., n] as MXFP4 holds it."""
    return decode(*encode(x), np.asarray(x).shape[-1])


def attn(q, k, v, lens, scale):
    """q [B, S, H, D] against the first lens[b] rows of k, v [B, n, heads, D];
    query head h reads key head h // (H // heads).  O [B, S, H, D], LSE
    [B, H, S], and the sum over keys of weight * |v| (for error bounds)."""
    B, S, H, D = q.shape
    G = H // k.shape[2]
    o, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full((B, H, S), -np.inf)
    for b in range(B):
        n = int(lens[b])
        for h in range(H if n > 0 else 0):
            s = q[b, :, h] @ k[b, :n, h // G].T * scale
            m = s.max(1, keepdims=True)
            p = np.exp(s - m)
            l = p.sum(1, keepdims=True)
            o[b, :, h] = p @ v[b, :n, h // G] / l
            mag[b, :, h] = p @ np.abs(v[b, :n, h // G]) / l
            lse[b, h] = (m + np.log(l))[:, 0]
    return o, lse, mag
