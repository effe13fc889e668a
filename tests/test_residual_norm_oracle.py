"""Pins of the seam's oracle (oracle/residual_norm.py) on the CPU: what norms
leave fixed, the identity without a branch, and every gradient against
differences of the forward definition."""
import numpy as np
import pytest

from oracle import residual_norm as rn


def test_norms():
    t = np.random.default_rng(0).standard_normal((5, 64)) * 3 + 1
    u, _ = rn.normalize(t, "layer", 0.0)
    assert np.allclose(u.mean(1), 0) and np.allclose(u.var(1), 1)
    assert np.allclose(rn.normalize(2 * t + 7, "layer", 0.0)[0], u)
    r, _ = rn.normalize(t, "rms", 0.0)
    assert np.allclose((r * r).mean(1), 1) and np.allclose(rn.normalize(5 * t, "rms", 0.0)[0], r)


def test_no_branch_is_the_stream():
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((4, 16)), rng.standard_normal((4, 16))
    xo, h = rn.forward(x, y, gate=np.zeros(16))
    assert np.array_equal(xo, x) and np.allclose(h, rn.normalize(x, "layer", 1e-6)[0])


@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("post", [None, "layer", "rms"])
@pytest.mark.parametrize("mod", [True, False])
def test_gradients_by_differences(norm, post, mod):
    rng = np.random.default_rng(2)
    rows, C, group = 5, 12, 2

    def r(*s):
        return rng.standard_normal(s)
    v = {"x": r(rows, C), "y": r(rows, C), "gate": r(3, C)}
    if mod:
        v["scale"], v["shift"] = r(3, C), r(3, C)
    else:
        v["w"] = r(C)
        if norm == "layer":
            v["b"] = r(C)
    if post:
        v["post_w"] = r(C)
        if post == "layer":
            v["post_b"] = r(C)
    gh, gx = r(rows, C), r(rows, C)
    how = {"norm": norm, "post": post, "group_rows": group, "alpha": 0.7, "eps": 1e-3}

    def loss(vals):
        xo, h = rn.forward(**vals, **how)
        return (h * gh).sum() + (xo * gx).sum()
    xo, _ = rn.forward(**v, **how)
    g = rn.backward(xo, v["y"], gh, gx, **{k: a for k, a in v.items() if k not in ("x", "y", "shift")}, **how)
    for name in v:
        for at in [tuple(rng.integers(0, n) for n in v[name].shape) for _ in range(6)]:
            d = 1e-6
            hi, lo = (dict(v, **{name: v[name].copy()}) for _ in range(2))
            hi[name][at] += d
            lo[name][at] -= d
            num = (loss(hi) - loss(lo)) / (2 * d)
            assert np.isclose(g["d" + name][at], num, rtol=1e-5, atol=1e-6), (name, at)
    assert all((np.abs(g[n]) <= g[f"|{n}|"] * (1 + 1e-9)).all() for n in g if not n.startswith("|"))
