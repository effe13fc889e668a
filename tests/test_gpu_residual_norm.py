"""GPU parity of the seam between two branches (regenvc_residual_norm_*)
against the fp64 oracle (oracle/residual_norm.py).

Bounds: a row's statistics are sums of C <= 8192 values, up to 32 in sequence
per lane and then a tree of 8: 40 roundings of 2^-24, and a few more for the
elementwise steps: within 2^-18 of the magnitudes that enter.  Sums over rows
add n 2^-24 for n rows in sequence (one wave's share).  A bf16 output adds half
a step, 2^-8.
"""
import numpy as np
import pytest

from oracle import residual_norm as orn
from paper_2607_28144_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
REL = 2.0 ** -18


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def dit():
    from paper_2607_28144_amd import dit as m
    return m


def host(t):
    return t.double().cpu().numpy()


def case(rows, C, norm="layer", post=None, mod=True, gate=True, group=0, f32=False, weights=True, seed=0):
    """The device tensors of a call, by argument name."""
    rng = np.random.default_rng(seed + rows + C)
    G = -(-rows // group) if group else 1

    def f(*shape, mean=0.0, std=1.0):
        return torch.from_numpy((rng.standard_normal(shape) * std + mean).astype(np.float32)).cuda()
    act = torch.float32 if f32 else torch.bfloat16
    t = {"x": f(rows, C, std=2.0, mean=0.5), "y": f(rows, C).to(act), "gh": f(rows, C).to(act), "gx": f(rows, C)}
    v = {}
    if gate:
        v["gate"] = f(G, C, std=0.5)
    if mod:
        v["scale"], v["shift"] = f(G, C, std=0.5), f(G, C, std=0.5)
    elif weights:
        v["w"] = f(C, mean=1.0, std=0.2).bfloat16()
        if norm == "layer":
            v["b"] = f(C, std=0.2).bfloat16()
    if post and weights:
        v["post_w"] = f(C, mean=1.0, std=0.2).bfloat16()
        if post == "layer":
            v["post_b"] = f(C, std=0.2).bfloat16()
    return t, v, {"norm": norm, "post": post, "group_rows": group}


def check(name, got, ref, tol):
    got = host(got)
    err = np.abs(got - ref)
    ratio = float((err / tol).max())
    assert got.shape == ref.shape and np.isfinite(got).all() and ratio <= 1.0, f"{name}: {ratio:.3f} of the bound"
    return ratio


def run(t, v, how, f32, alpha=0.75):
    rows, C = t["x"].shape
    n = {k: host(a) for k, a in v.items()}
    x, y = host(t["x"]), host(t["y"])
    half = 2.0 ** -22 if f32 else 2.0 ** -8
    xo, h = dit().residual_norm_fwd(t["x"], t["y"], alpha=alpha, **v, **how)
    rx, rh = orn.forward(x, y, alpha=alpha, **n, **how)
    # magnitudes: of the stream's sum, and of a unit value with its mean
    zero = np.zeros((rows, 1))
    mu_y, s_y = (y.mean(1, keepdims=True), y.std(1, keepdims=True) + 1e-3) if how["post"] else (zero, zero + 1)
    au = (np.abs(y) + np.abs(mu_y)) / s_y * 4 + 4
    g = np.abs(orn._rows(n.get("gate"), rows, how["group_rows"], 1.0))
    ax = alpha * np.abs(x) + g * au * np.abs(n.get("post_w", 1.0)) + g * np.abs(n.get("post_b", 0.0))
    r1 = check("x'", xo, rx, REL * ax)
    # h follows from x' as it is stored: the oracle starts from that
    _, rh = orn.forward(host(xo), np.zeros_like(y), gate=None, alpha=1.0, **{k: a for k, a in n.items() if k in (
        "scale", "shift", "w", "b")}, norm=how["norm"], group_rows=how["group_rows"])
    unit, sigma = orn.normalize(host(xo), how["norm"], 1e-6)
    an = np.abs(unit) + np.abs(host(xo)).mean(1, keepdims=True) / sigma + 1
    mul = 1 + np.abs(orn._rows(n.get("scale"), rows, how["group_rows"], 0.0)) if "scale" in n else np.abs(n.get("w", 1.0))
    add = np.abs(orn._rows(n.get("shift"), rows, how["group_rows"], 0.0)) if "shift" in n else np.abs(n.get("b", 0.0))
    r2 = check("h", h, rh, REL * (an * mul + add) + half * np.abs(rh))
    # backward, from a stream that is not the forward's, so that both halves are tested alone
    b = {k: a for k, a in v.items() if k != "shift"}
    got = dit().residual_norm_bwd(t["x"], t["y"], t["gh"], t["gx"], alpha=alpha, **b, **how)
    ref = orn.backward(x, y, host(t["gh"]), host(t["gx"]), alpha=alpha, **{k: a for k, a in n.items() if k != "shift"},
                       **how)
    worst = 0.0
    for name in got._fields:
        z = getattr(got, name)
        assert (z is None) == (name not in ref), name
        if z is not None:
            tol = 4 * REL * ref[f"|{name}|"] + (half * np.abs(ref[name]) if name == "dy" else 0)
            if name not in ("dx", "dy"):
                tol = tol + rows * 2.0 ** -24 * ref[f"|{name}|"]
            worst = max(worst, check(name, z, ref[name], tol + 1e-30))
    print(f"[seam] rows={rows} C={C} {how}: x' {r1:.3f} h {r2:.3f} gradients {worst:.3f} of their bounds", flush=True)


@pytest.mark.parametrize("rows,C", [(1, 8), (3, 512), (5, 520), (2, 1024), (17, 1536), (4, 2048), (3, 2056), (2, 4096),
                                    (3, 6144), (2, 8192), (301, 264)])
@pytest.mark.parametrize("f32", [False, True])
def test_widths(rows, C, f32):
    t, v, how = case(rows, C, "layer", "rms", f32=f32)
    run(t, v, how, f32)


@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("post", [None, "layer", "rms"])
@pytest.mark.parametrize("mod,gate,weights", [(True, True, True), (False, True, True), (False, False, False)])
def test_forms(norm, post, mod, gate, weights):
    for C in (1536, 2560):
        t, v, how = case(37, C, norm, post, mod, gate, weights=weights)
        run(t, v, how, False)


@pytest.mark.parametrize("rows,group", [(10, 3), (10, 1), (10, 10), (10, 99), (700, 1), (3000, 1000), (2000, 700)])
def test_groups(rows, group):
    """Groups that end ragged, one row each, more than there are workgroups, larger than the batch."""
    t, v, how = case(rows, 512, "layer", "layer", mod=group != 10, group=group)
    if group >= rows:
        v = {k: a[0] if k in ("gate", "scale", "shift") else a for k, a in v.items()}
    run(t, v, how, False)
    if group >= rows:
        assert dit().residual_norm_bwd(t["x"], t["y"], t["gh"], gate=v.get("gate"), group_rows=group).dgate.shape == (1, 512)


def test_vectors_as_slices_of_a_modulation():
    """gate, scale and shift as column ranges of one [groups, 6 C] tensor; strided rows of everything else."""
    rows, C, group = 50, 512, 20
    t, v, how = case(rows, C, "rms", "rms", group=group)
    m = torch.randn(3, 6 * C, device="cuda")
    for i, n in enumerate(("gate", "scale", "shift")):
        m[:, i * C:(i + 1) * C] = v[n]
        v[n] = m[:, i * C:(i + 1) * C]
    run(t, v, how, False)

    def wide(a):
        w = torch.full((a.shape[0], C + 24), float("nan"), dtype=a.dtype, device="cuda")
        w[:, 8:8 + C] = a
        return w[:, 8:8 + C]
    xo, h = dit().residual_norm_fwd(t["x"], t["y"], **v, **how)
    xs, hs = dit().residual_norm_fwd(wide(t["x"]), wide(t["y"]), out=wide(xo * 0), h=wide(h * 0), **v, **how)
    assert torch.equal(xo, xs) and torch.equal(h, hs)
    v.pop("shift")
    a = dit().residual_norm_bwd(t["x"], t["y"], t["gh"], t["gx"], **v, **how)
    b = dit().residual_norm_bwd(wide(t["x"]), wide(t["y"]), wide(t["gh"]), wide(t["gx"]), **v, **how)
    for p, q in zip(a, b):
        assert (p is None and q is None) or torch.equal(p, q)


def test_in_place_and_surroundings():
    rows, C = 40, 1536
    t, v, how = case(rows, C)
    xo, h = dit().residual_norm_fwd(t["x"], t["y"], **v, **how)
    x = torch.full((rows + 2, C), 3.0, device="cuda")
    x[1:-1] = t["x"]
    dit().residual_norm_fwd(x[1:-1], t["y"], out=x[1:-1], **v, **how)
    assert torch.equal(x[1:-1], xo) and bool((x[0] == 3.0).all()) and bool((x[-1] == 3.0).all())
    v.pop("shift")
    g = dit().residual_norm_bwd(t["x"], t["y"], t["gh"], t["gx"], **v, **how)
    gx = t["gx"].clone()
    g2 = dit().residual_norm_bwd(t["x"], t["y"], t["gh"], gx, dx=gx, **v, **how)
    assert torch.equal(g.dx, gx) and all(torch.equal(a, b) for a, b in zip(g, g2) if a is not None)
    none = dit().residual_norm_bwd(t["x"], t["y"], t["gh"], None, **v, **how)
    zero = dit().residual_norm_bwd(t["x"], t["y"], t["gh"], torch.zeros_like(gx), **v, **how)
    assert torch.equal(none.dx, zero.dx) and torch.equal(none.dy, zero.dy)


def test_nonfinite_rows_stay_alone():
    rows, C = 20, 1536
    t, v, how = case(rows, C, "layer", "rms")
    xo, h = dit().residual_norm_fwd(t["x"], t["y"], **v, **how)
    t["x"][3, 7] = float("inf")
    t["y"][5, 9] = float("nan")
    xo2, h2 = dit().residual_norm_fwd(t["x"], t["y"], **v, **how)
    ok = torch.ones(rows, dtype=torch.bool, device="cuda")
    ok[3] = ok[5] = False
    assert torch.equal(h[ok], h2[ok]) and torch.equal(xo[ok], xo2[ok])
    assert bool(torch.isnan(h2[3]).any()) and bool(torch.isnan(h2[5]).all())


def test_no_rows():
    C = 512
    x, y = torch.empty(0, C, device="cuda"), torch.empty(0, C, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(C, device="cuda", dtype=torch.bfloat16)
    xo, h = dit().residual_norm_fwd(x, y, w=w)
    assert xo.shape == h.shape == (0, C)
    g = dit().residual_norm_bwd(x, y, y, w=w, gate=torch.ones(C, device="cuda"))
    assert bool((g.dw == 0).all()) and bool((g.dgate == 0).all())


def test_differences():
    """The gradients against differences of the forward kernel (float32 throughout): the directional derivative of
    L = <h, gh> + <x', gx> along a random direction of every input."""
    rows, C = 6, 512
    t, v, how = case(rows, C, "layer", "layer", f32=True, group=4)
    v = {k: a for k, a in v.items()}
    xo, _ = dit().residual_norm_fwd(t["x"], t["y"], **v, **how)
    b = {k: a for k, a in v.items() if k != "shift"}
    g = dit().residual_norm_bwd(xo, t["y"], t["gh"], t["gx"], **b, **how)
    names = {"x": "dx", "y": "dy", "gate": "dgate", "scale": "dscale", "shift": "dshift"}
    torch.manual_seed(0)
    for name, grad in names.items():
        base = t[name] if name in t else v[name]
        d = torch.randn_like(base)

        def loss(eps):
            tt, vv = dict(t), dict(v)
            (tt if name in t else vv)[name] = base + eps * d
            xo_, h_ = dit().residual_norm_fwd(tt["x"], tt["y"], **vv, **how)
            return float((h_.double() * t["gh"].double()).sum() + (xo_.double() * t["gx"].double()).sum())
        # central difference: truncation of order eps^2, rounding 2^-22 sqrt(rows C) |h| / eps
        eps = 2.0 ** -6
        num = (loss(eps) - loss(-eps)) / (2 * eps)
        ana = float((getattr(g, grad).double() * d.double()).sum())
        size = float((getattr(g, grad).double() * d.double()).square().sum().sqrt())
        assert abs(num - ana) <= 0.02 * size + 0.01, (name, num, ana, size)


def test_backward_captured():
    """The backward pass in a graph, replayed between eager calls, bitwise as those."""
    t, v, how = case(500, 1536, "layer", "rms", group=200)
    v.pop("shift")
    ref = dit().residual_norm_bwd(t["x"], t["y"], t["gh"], t["gx"], **v, **how)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = dit().residual_norm_bwd(t["x"], t["y"], t["gh"], t["gx"], **v, **how)
    for _ in range(3):
        for z in out:
            if z is not None:
                z.zero_()
        graph.replay()
        eager = dit().residual_norm_bwd(t["x"], t["y"], t["gh"], t["gx"], **v, **how)
        torch.cuda.synchronize()
        for a, b, c in zip(ref, out, eager):
            assert a is None or (torch.equal(a, b) and torch.equal(a, c))
