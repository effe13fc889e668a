"""Reference oracle of the seam between two branches of a block, forward and
backward -- TEST INFRASTRUCTURE ONLY: plain float64 numpy definitions, nothing
shared with the product.

    u  = N_post(y) w_post + b_post     (or y)
    x' = alpha x + gate u
    h  = N_pre(x') mul + add           mul = 1 + scale, add = shift, or mul = w, add = b

with a row's vectors taken from its group (row // group_rows).
"""
from __future__ import annotations

import numpy as np


def normalize(t, kind, eps):
    """The unit row values, and sigma (or rms) [rows, 1]."""
    z = t - t.mean(1, keepdims=True) if kind == "layer" else t
    sigma = np.sqrt((z * z).mean(1, keepdims=True) + eps)
    return z / sigma, sigma


def normalize_grad(g, unit, sigma, kind):
    """The gradient of t, given that of its unit values."""
    g = g - unit * (g * unit).mean(1, keepdims=True) - (g.mean(1, keepdims=True) if kind == "layer" else 0)
    return g / sigma


def _rows(v, rows, group_rows, missing):
    if v is None:
        return missing
    v = np.atleast_2d(v)
    return v[np.arange(rows) // group_rows] if group_rows else v[np.zeros(rows, int)]


def forward(x, y, norm="layer", post=None, gate=None, scale=None, shift=None, w=None, b=None, post_w=None, post_b=None,
            alpha=1.0, eps=1e-6, group_rows=0):
    rows = x.shape[0]
    u = y
    if post is not None:
        u = normalize(y, post, eps)[0] * (1 if post_w is None else post_w) + (0 if post_b is None else post_b)
    xo = alpha * x + _rows(gate, rows, group_rows, 1.0) * u
    mul = 1 + _rows(scale, rows, group_rows, 0.0) if scale is not None else 1 if w is None else w
    add = _rows(shift, rows, group_rows, 0.0) if shift is not None else 0 if b is None else b
    return xo, normalize(xo, norm, eps)[0] * mul + add


def backward(xo, y, gh, gx, norm="layer", post=None, gate=None, scale=None, w=None, b=None, post_w=None, post_b=None,
             alpha=1.0, eps=1e-6, group_rows=0):
    """A dict of gradients, each with the sum of its terms' magnitudes (for error bounds) under '|name|'."""
    rows, C = xo.shape
    group = np.arange(rows) // group_rows if group_rows else np.zeros(rows, int)
    G = int(group[-1]) + 1

    def per_group(t):
        out = np.zeros((G, C))
        np.add.at(out, group, t)
        return out
    unit, sigma = normalize(xo, norm, eps)
    mul = 1 + _rows(scale, rows, group_rows, 0.0) if scale is not None else 1 if w is None else w
    g = gh * mul
    dr = (0 if gx is None else gx) + normalize_grad(g, unit, sigma, norm)
    # magnitudes of what is added up
    a_dr = (0 if gx is None else np.abs(gx)) + (np.abs(g) + np.abs(g).mean(1, keepdims=True)
                                                + np.abs(unit) * np.abs(g * unit).mean(1, keepdims=True)) / sigma
    ga = _rows(gate, rows, group_rows, 1.0)
    du, a_du = ga * dr, np.abs(ga) * a_dr
    out = {"dx": alpha * dr, "|dx|": abs(alpha) * a_dr}
    if post is None:
        u, a_u = y, np.abs(y)
        out["dy"], out["|dy|"] = du, a_du
    else:
        pu, ps = normalize(y, post, eps)
        pw = 1 if post_w is None else post_w
        a_p = np.abs(pu) + 1
        u, a_u = pu * pw + (0 if post_b is None else post_b), a_p * np.abs(pw) + (0 if post_b is None else np.abs(post_b))
        q = du * pw
        out["dy"] = normalize_grad(q, pu, ps, post)
        aq = a_du * np.abs(pw)
        out["|dy|"] = (aq + aq.mean(1, keepdims=True) + a_p * (aq * a_p).mean(1, keepdims=True)) / ps
        if post_w is not None:
            out["dpost_w"], out["|dpost_w|"] = (du * pu).sum(0), (a_du * a_p).sum(0)
        if post_b is not None:
            out["dpost_b"], out["|dpost_b|"] = du.sum(0), a_du.sum(0)
    if gate is not None:
        out["dgate"], out["|dgate|"] = per_group(dr * u), per_group(a_dr * a_u)
    a_n = np.abs(gh) * (np.abs(unit) + 1)
    if scale is not None:
        out["dscale"], out["|dscale|"] = per_group(gh * unit), per_group(a_n)
        out["dshift"], out["|dshift|"] = per_group(gh), per_group(np.abs(gh))
    if w is not None:
        out["dw"], out["|dw|"] = (gh * unit).sum(0), a_n.sum(0)
    if b is not None:
        out["db"], out["|db|"] = gh.sum(0), np.abs(gh).sum(0)
    return out
