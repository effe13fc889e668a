"""GPU parity of the append to a cache in pages (norm of heads, rotation, mean
keys) against the fp64 oracle (oracle/paged.py).

Bounds.  One rounding to bf16: 2^-8 of the value.  Before it, in fp32: the norm
within 24 roundings (a sum of D squares by 8, then log2(D / 8) exchanges, a
division, a root, a reciprocal, two products), and a rotation whose angle is exact
to 2^-25 turns (1.9e-7 rad) and whose sine and cosine are the hardware's, taken as
within 1.5e-6; both relative to the length of the rotated pair.  The mean key of a
page is that of the keys as the kernel stored them, rounded once from 64 bits: equal.
"""
import numpy as np
import pytest

from oracle import dit as odit
from oracle import paged as opaged
from paged_cases import Case
from paper_2607_28144_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def paged():
    from paper_2607_28144_amd import paged as m
    return m


def bf16(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).cuda()


def host(t):
    return t.double().cpu().numpy()


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def inside(name, got, ref, pair):
    tol = 2.0 ** -8 * np.abs(ref) + (2e-6 + 24 * 2.0 ** -24) * pair + 1e-38
    err = np.abs(got - ref)
    print(f"[paged append] {name}: max|d|={err.max():.3e} ({(err / tol).max():.3f} of the bound)", flush=True)
    assert (err <= tol).all()


def pairs_of(x, rot, layout):
    """The length of the pair that each channel of x [..., D] is rotated in (its own size where it is not)."""
    y = np.abs(x).copy()
    if rot:
        i0, i1 = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if layout == "interleaved" else \
            (np.arange(rot // 2), rot // 2 + np.arange(rot // 2))
        y[..., i0] = y[..., i1] = np.hypot(x[..., i0], x[..., i1])
    return y


def pool(c, old=7):
    """Pools of old values, and the tensors of a call's sequences."""
    rng = np.random.default_rng(old)
    k, v = (synth.normal_bf16(rng, c.k.shape) for _ in range(2))
    means = synth.normal_bf16(rng, (c.k.shape[0], c.heads, c.D))
    return k, v, means


# rows, lens, H, heads, D, page
CASES = [([1], [1], 1, 1, 64, 16), ([1], [300], 12, 12, 128, 64), ([1, 1, 1], [17, 1, 900], 16, 4, 64, 16),
         ([100, 3, 0, 30], [100, 66, 9, 700], 5, 1, 128, 32), ([65, 64], [65, 320], 3, 3, 64, 128),
         ([40], [33], 2, 2, 128, 16), ([1] * 70, list(range(70, 140)), 2, 1, 64, 1024)]


@pytest.mark.parametrize("rows,lens,H,heads,D,page", CASES)
@pytest.mark.parametrize("layout,rot,norm,means", [("half", 1.0, True, True), ("interleaved", 1.0, False, False),
                                                   ("half", 0.5, False, True), ("interleaved", 0.25, True, False),
                                                   ("half", 0.25, True, True),
                                                   ("none", 0, True, True), ("none", 0, False, False)])
def test_append(rows, lens, H, heads, D, page, layout, rot, norm, means):
    c = Case(rows, lens, H, heads, D, page, seed=sum(lens) + H, lead=1, tail=2)
    rng = np.random.default_rng(H)
    wide = synth.normal_bf16(rng, (c.T, H + 2 * heads, D), 2.0)
    wq, wk = synth.normal_bf16(rng, (D,)), synth.normal_bf16(rng, (D,))
    k0, v0, m0 = pool(c)
    cache = paged().PagedCache(bf16(k0), bf16(v0), bf16(m0) if means else None)
    rot = int(rot * D)
    rotary = paged().Rotary(rot, layout=layout) if rot else None
    t = bf16(wide)
    got = torch.full((c.T, H, D), 5.0, dtype=torch.bfloat16, device="cuda")
    w = {"w_q": bf16(wq), "w_k": bf16(wk)} if norm else {}
    table, first, n = ints(c.table), ints(c.first), ints(c.lens)
    paged().append(cache, table, first, n, t[:, H:H + heads], t[:, H + heads:], q=t[:, :H], rotary=rotary, q_out=got, **w)
    x = odit.widen(wide)
    turns = rotary.turns.cpu().numpy() if rot else ()
    args = dict(w_q=odit.widen(wq) if norm else None, w_k=odit.widen(wk) if norm else None)
    ref, rk, rv, written = opaged.append(x[:, :H], x[:, H:H + heads], x[:, H + heads:], odit.widen(k0), odit.widen(v0), c.table,
                                         c.first, c.lens, turns=turns, layout=layout, **args)
    live = slice(1, c.T - 2)
    name = f"{(rows[:4], lens[:4], H, heads, D, page, layout, rot, norm)}"
    inside(name + " q", host(got)[live], ref[live], pairs_of(ref[live], rot, layout))
    assert bool((got[:1] == 5.0).all()) and bool((got[c.T - 2:] == 5.0).all())
    gk = host(cache.k)
    at = np.broadcast_to(written[:, None, :, None], rk.shape)
    inside(name + " k", np.where(at, gk, 0), np.where(at, rk, 0), pairs_of(np.where(at, rk, 0), rot, layout))
    assert np.array_equal(np.where(at, 0, gk), np.where(at, 0, odit.widen(k0)))
    assert np.array_equal(host(cache.v), rv)
    if means:
        ref_m = odit.round_bf16(opaged.means(gk, c.table, c.first, c.lens, odit.widen(m0)))
        assert np.array_equal(host(cache.means), ref_m)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_places(layout):
    """Places near 2^29: the angle's whole turns are taken off in 64 bits.  (A table of one column short of all of
    them: only q shows the rotation, and a k whose page does not exist is not stored.)"""
    H, D, n = 2, 64, 3
    place = (1 << 29) - 5
    rng = np.random.default_rng(3)
    q = synth.normal_bf16(rng, (n, H, D))
    cache = paged().PagedCache.zeros(1, 1024, H, D)
    rotary = paged().Rotary(D, layout=layout)
    x = bf16(q)
    got = paged().append(cache, ints([[0]]), ints([0, n]), ints([place + n]), x, x, q=x, rotary=rotary)
    ref = np.stack([opaged.rotate(odit.widen(q[i]), place + i, rotary.turns.cpu().numpy(), layout) for i in range(n)])
    inside(f"far {layout}", host(got), ref, pairs_of(ref, D, layout))
    assert bool((cache.k == 0).all()) and bool((cache.v == 0).all())


def test_in_place_and_without_q():
    """q_out = q within a fused projection; keys and values alone; no sequences; no heads of queries."""
    c = Case([30, 5], [40, 100], 4, 2, 128, 16, seed=8)
    rng = np.random.default_rng(2)
    wide = bf16(synth.normal_bf16(rng, (c.T, 8, 128)))
    k0, v0, m0 = pool(c)
    table, first, n = ints(c.table), ints(c.first), ints(c.lens)
    w = {"w_q": bf16(synth.normal_bf16(rng, (128,))), "w_k": bf16(synth.normal_bf16(rng, (128,)))}
    rot = paged().Rotary(128)
    a = paged().PagedCache(bf16(k0), bf16(v0), bf16(m0))
    ref = paged().append(a, table, first, n, wide[:, 4:6], wide[:, 6:], q=wide[:, :4], rotary=rot, **w)
    b = paged().PagedCache(bf16(k0), bf16(v0), bf16(m0))
    keep = wide.clone()
    out = paged().append(b, table, first, n, wide[:, 4:6], wide[:, 6:], q=wide[:, :4], q_out=wide[:, :4], rotary=rot, **w)
    assert torch.equal(out, ref) and torch.equal(wide[:, 4:], keep[:, 4:])
    d = paged().PagedCache(bf16(k0), bf16(v0), bf16(m0))
    assert paged().append(d, table, first, n, wide[:, 4:6], wide[:, 6:], rotary=rot, w_k=w["w_k"]) is None
    for p in (b, d):
        assert torch.equal(p.k, a.k) and torch.equal(p.v, a.v) and torch.equal(p.means, a.means)
    paged().append(d, table[:0], first[:1], n[:0], wide[:0, 4:6], wide[:0, 6:], q=wide[:0, :4])
    assert torch.equal(d.k, a.k)


def test_pages_that_do_not_exist_and_places_before_the_first():
    """Tokens of negative places, of pages outside the pool and past the table are not stored; the rest is."""
    c = Case([40, 40, 20], [20, 100, 60], 2, 2, 64, 16, seed=5)
    c.table[1, 4], c.table[2, 3] = c.k.shape[0], -1
    table = c.table[:, :6]
    lens = np.array([20, 100, 60], np.int32)
    rng = np.random.default_rng(2)
    x = synth.normal_bf16(rng, (c.T, 2, 64))
    k0, v0, m0 = pool(c)
    cache = paged().PagedCache(bf16(k0), bf16(v0), bf16(m0))
    q = paged().append(cache, ints(table), ints(c.first), ints(lens), bf16(x), bf16(x), q=bf16(x))
    _, rk, rv, _ = opaged.append(None, odit.widen(x), odit.widen(x), odit.widen(k0), odit.widen(v0), table, c.first, lens)
    assert np.array_equal(host(cache.k), rk) and np.array_equal(host(cache.v), rv) and torch.equal(q, bf16(x))
    assert np.array_equal(host(cache.means), odit.round_bf16(opaged.means(rk, table, c.first, lens, odit.widen(m0))))
