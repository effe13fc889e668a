"""Pins of the MXFP4 oracle (oracle/mx.py) on the CPU: the sixteen codes by
hand, rounding and scale by search over all representable values, attention
against its two-key closed form."""
import math

import numpy as np

from oracle import mx


def test_every_value_of_the_grid_is_itself():
    for e in (-100, -1, 0, 7, 90):
        x = np.ldexp(np.concatenate([mx.GRID, -mx.GRID, np.zeros(16)]), e)
        assert np.array_equal(mx.values(x), x)
        code, byte = mx.encode(x)
        assert byte[0] == e + 127 and list(code[0, :8]) == list(range(8)) and list(code[0, 9:16]) == list(range(9, 16))


def test_rounding_by_hand():
    """Ties go to the even code; beyond 6 all is 6."""
    x = np.zeros(32)
    pairs = [(0.25, 0.0), (0.75, 1.0), (1.25, 1.0), (1.75, 2.0), (2.5, 2.0), (3.5, 4.0), (5.0, 4.0), (5.01, 6.0),
             (7.9, 6.0), (0.26, 0.5), (-1.75, -2.0), (-5.0, -4.0), (4.0, 4.0)]
    for i, (a, _) in enumerate(pairs):
        x[i] = a
    assert list(mx.values(x)[: len(pairs)]) == [b for _, b in pairs]


def test_nearest_by_search():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 32)) * np.exp(rng.standard_normal((200, 1)) * 5)
    v = mx.values(x)
    for row, val in zip(x, v):
        s = 2.0 ** (math.floor(math.log2(np.abs(row).max())) - 2)
        grid = np.concatenate([mx.GRID, -mx.GRID]) * s
        assert np.isin(val, grid).all()
        assert np.allclose(np.abs(row - val), np.abs(row[:, None] - grid).min(1), rtol=0, atol=0)


def test_small_zero_and_nonfinite_blocks():
    x = np.zeros((4, 40))
    x[0, 3] = 2.0 ** -133          # below the least scale's half step: 0
    x[1, 3] = 2.0 ** -126          # 2 units of 2^-127
    x[2, 35] = np.inf
    x[3, 0] = np.nan
    code, byte = mx.encode(x)
    assert byte[0, 0] == 0 and byte[1, 0] == 0 and code[1, 0, 3] == 4 and byte[2, 1] == 255 and byte[3, 0] == 255
    v = mx.values(x)
    assert v[0, 3] == 0 and v[1, 3] == 2.0 ** -126
    assert np.isnan(v[2, 32:]).all() and (v[2, :32] == 0).all() and np.isnan(v[3, :32]).all()


def test_attention_of_two_places():
    """O = v0 + sigmoid(s1 - s0)(v1 - v0); grouped heads read their key head; no place: 0 and -inf."""
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((2, 3, 4, 8)), rng.standard_normal((2, 5, 2, 8)), rng.standard_normal((2, 5, 2, 8))
    o, lse, mag = mx.attn(q, k, v, [2, 0], 0.3)
    for s in range(3):
        for h in range(4):
            a, b = (0.3 * float(q[0, s, h] @ k[0, j, h // 2]) for j in range(2))
            w = 1 / (1 + math.exp(a - b))
            assert np.allclose(o[0, s, h], v[0, 0, h // 2] * (1 - w) + v[0, 1, h // 2] * w)
            assert np.allclose(mag[0, s, h], np.abs(v[0, 0, h // 2]) * (1 - w) + np.abs(v[0, 1, h // 2]) * w)
            assert math.isclose(lse[0, h, s], math.log(math.exp(a) + math.exp(b)))
    assert (o[1] == 0).all() and np.isneginf(lse[1]).all()
