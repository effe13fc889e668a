"""Pins of the paged cache's oracle and of the rotary tables, on the CPU: brute
loops, closed forms and invariances."""
import math

import numpy as np
import pytest

from oracle import dit as odit
from oracle import paged as opaged
from paged_cases import Case

torch = pytest.importorskip("torch")


def test_attention_is_dense_attention():
    """Gathered by hand into dense keys: the same O and LSE, causal and not."""
    c = Case([5, 0, 3], [37, 10, 3], 4, 2, 64, 16, seed=1, lead=2, tail=1)
    q, k, v = c.wide()
    for causal in (True, False):
        o, lse, mag, _ = opaged.attn(q, k, v, c.table, c.first, c.lens, causal, 0.125)
        assert np.isnan(o[:2]).all() and np.isnan(o[-1]).all()
        for b, n in ((0, 37), (2, 3)):
            f0, f1 = c.first[b], c.first[b + 1]
            for t in range(f0, f1):
                see = n - (f1 - t) + 1 if causal else n
                for h in range(4):
                    kk = np.array([k[c.table[b, p // 16], h // 2, p % 16] for p in range(see)])
                    vv = np.array([v[c.table[b, p // 16], h // 2, p % 16] for p in range(see)])
                    s = np.exp(kk @ q[t, h] * 0.125)
                    assert np.allclose(o[t, h], s @ vv / s.sum(), rtol=1e-12) and np.isclose(lse[h, t], math.log(s.sum()))
                    assert (mag[t, h] >= np.abs(o[t, h]) - 1e-12).all()


def test_all_pages_selected_is_dense_and_none_is_empty():
    c = Case([9, 1], [50, 70], 2, 1, 64, 16, seed=2)
    q, k, v = c.wide()
    dense = opaged.attn(q, k, v, c.table, c.first, c.lens, True, 0.1)
    every = np.tile(np.arange(5, dtype=np.int32), (10 // 4 + 2, 1, 1))
    same = opaged.attn(q, k, v, c.table, c.first, c.lens, True, 0.1, every, 4)
    assert np.allclose(dense[0], same[0]) and np.allclose(dense[1], same[1])
    none = opaged.attn(q, k, v, c.table, c.first, c.lens, True, 0.1, np.full_like(every, -1), 4)
    assert (none[0] == 0).all() and np.isneginf(none[1]).all()


def test_selection_by_hand():
    table, page = np.arange(6, dtype=np.int32)[None], 16
    means = np.zeros((6, 1, 64))
    means[:, 0, 0] = [0.0, 5.0, -1.0, 5.0, 2.0, 9.0]
    q = np.zeros((3, 2, 64))
    q[:, :, 0] = 1.0
    args = (q, means, table, [0, 3], [96], page)
    pick = lambda *a: opaged.select(*args, *a)[:, 0].tolist()  # noqa: E731
    assert pick(2, 4, 0, 0, False) == [[1, 5]]
    assert pick(2, 4, 1, 0, False) == [[0, 5]]
    assert pick(3, 4, 0, 1, False) == [[1, 3, 5]]
    assert pick(2, 4, 0, 1, False) == [[1, 5]]           # 1 and 3 tie: the lower page
    assert pick(8, 4, 0, 0, False) == [[0, 1, 2, 3, 4, 5, -1, -1]]
    assert pick(1, 1, 0, 0, True) == [[5], [5], [5], [-1]]
    assert opaged.select(q, means, table, [0, 3], [82], page, 1, 1, 0, 0, True)[:, 0].tolist() == [[1], [5], [5], [-1]]


def test_rotation_keeps_lengths_and_differences():
    """A rotation keeps each pair's length, and the product of a query and a key depends on the places' difference."""
    rng = np.random.default_rng(0)
    from paper_2607_28144_amd import paged
    for layout in ("half", "interleaved"):
        turns = paged.Rotary(32, layout=layout, device="cpu").turns.numpy()
        x, y = rng.standard_normal((2, 1, 64))
        for p in (0, 1, 1000, 1 << 20):
            z = opaged.rotate(x, p, turns, layout)
            assert np.isclose((z * z).sum(), (x * x).sum()) and np.array_equal(z[:, 32:], x[:, 32:])
        dot = lambda a, b: float((opaged.rotate(x, a, turns, layout) * opaged.rotate(y, b, turns, layout)).sum())  # noqa: E731
        assert np.isclose(dot(7, 3), dot(104, 100)) and not np.isclose(dot(7, 3), dot(7, 4))
        assert np.allclose(opaged.rotate(x, 0, turns, layout), x)


def test_layouts_are_permutations_of_one_another():
    rng = np.random.default_rng(1)
    from paper_2607_28144_amd import paged
    turns = paged.Rotary(64, device="cpu").turns.numpy()
    x = rng.standard_normal((3, 64))
    order = np.arange(64).reshape(2, 32).T.reshape(-1)  # channel of the half layout at each of the interleaved one
    a, b = opaged.rotate(x, 17, turns, "half"), opaged.rotate(x[:, order], 17, turns, "interleaved")
    assert np.allclose(a[:, order], b)


def test_rotary_tables():
    from paper_2607_28144_amd import paged
    r = lambda **kw: paged.Rotary(64, theta=10000.0, device="cpu", **kw)  # noqa: E731
    base = r()
    i = np.arange(32)
    assert np.allclose(base.turns.numpy() * 2 * np.pi, 10000.0 ** (-2 * i / 64), rtol=1e-14) and base.amplitude == 1.0
    assert base.turns.dtype == torch.float64
    lin = r(scaling="linear", factor=4.0)
    assert torch.allclose(lin.turns * 4, base.turns, rtol=1e-14)
    b = r(scaling="base", factor=8.0)
    assert b.turns[0] == base.turns[0] and np.isclose(float(base.turns[-1] / b.turns[-1]), 8.0)  # the last pair: factor times as slow
    p = r(scaling="parts", factor=8.0, original_len=4096)
    n = base.turns.numpy() * 4096
    assert np.array_equal(p.turns[n >= 32].numpy(), base.turns[n >= 32].numpy())
    assert np.allclose(p.turns[n <= 1].numpy() * 8, base.turns[n <= 1].numpy(), rtol=1e-14)
    mid = (n > 1) & (n < 32)
    assert mid.any() and (p.turns[mid] < base.turns[mid]).all() and (p.turns[mid] * 8 > base.turns[mid]).all()
    assert np.isclose(p.amplitude, 1 + 0.1 * math.log(8))
    assert r(scaling="parts", factor=1.0, original_len=10).amplitude == 1.0
    assert paged.Rotary(0, device="cpu").turns.numel() == 0
    for bad in ({"layout": "x"}, {"scaling": "x"}, {"factor": 2.0}, {"scaling": "parts", "factor": 2.0},
                {"scaling": "linear", "factor": 0.0}, {"scaling": "parts", "factor": 0.5, "original_len": 9},
                {"scaling": "parts", "factor": 2.0, "original_len": 9, "fast": 1.0}):
        with pytest.raises(ValueError):
            r(**bad)
    for dim in (-16, 8, 20):
        with pytest.raises(ValueError):
            paged.Rotary(dim, device="cpu")


def test_append_and_means_by_hand():
    c = Case([3, 2], [18, 2], 1, 1, 64, 16, seed=3)
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 1, 64))
    zero = np.zeros(c.k.shape)
    out, pk, pv, written = opaged.append(x, x, -x, zero, zero, c.table, c.first, c.lens, w_q=np.full(64, 2.0), eps=0.0)
    assert np.allclose((out ** 2).mean(-1), 4.0)
    assert written.sum() == 5 and written[c.table[0, 0], 15] and written[c.table[0, 1], :2].all() and written[c.table[1, 0], :2].all()
    assert np.array_equal(pk[c.table[0, 0], 0, 15], x[0, 0]) and np.array_equal(pv[c.table[0, 1], 0, 1], -x[2, 0])
    m = opaged.means(pk, c.table, c.first, c.lens, np.full((len(pk), 1, 64), 9.0))
    assert np.allclose(m[c.table[0, 0], 0], x[0, 0] / 16) and np.allclose(m[c.table[0, 1], 0], x[1:3, 0].mean(0))
    assert np.allclose(m[c.table[1, 0], 0], x[3:, 0].mean(0)) and (np.delete(m, c.table[[0, 0, 1], [0, 1, 0]], 0) == 9.0).all()


def test_case_marks_every_place_once():
    c = Case([4, 1, 0], [33, 16, 0], 1, 1, 64, 16)
    assert c.keep.sum() == 49 and np.isnan(odit.widen(c.k)).sum() == (c.keep.size - 49) * 64
    used = c.table[c.table >= 0]
    assert len(set(used.tolist())) == len(used) == 4
