"""GPU parity of attention over a bf16 cache in pages, and of the choice of
pages, against the fp64 oracle (oracle/paged.py).

Bounds.  A score q.k is a sum of D exact products in fp32: off by at most 12 *
2^-24 sum |q||k| (D / 32 additions of 32-deep sums, each within 2 roundings, and
one more for D = 64's order), times scale; the exponent's argument is rounded
twice more, relative to its size, and the exponential itself is within 2^-22.
Call that es, the largest over a row's keys.  Weights are rounded to bf16 (half a
step, 2^-8) and O is divided by the sum of the rounded weights, so |dO| <= (2^-8
+ 2 es)(sum p|v| + |O|), plus the output's own rounding; LSE takes unrounded
weights: es, and the roundings of a sum of n terms in lanes of n / 8.

The choice of pages is that of exact scores: it has to be equal.
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


def held(c, means=None):
    """The cache and the three arrays of a case's sequences."""
    return paged().PagedCache(bf16(c.k), bf16(c.v), means), ints(c.table), ints(c.first), ints(c.lens)


def check(name, o, lse, c, causal, scale=None, selected=None, q_block=1, f32=False):
    q, k, v = c.wide()
    scale = synth.default_scale(c.D) if scale is None else scale
    ro, rl, mag, big = opaged.attn(q, k, v, c.table, c.first, c.lens, causal, scale, selected, q_block)
    es = big * 14 * 2.0 ** -24 + 2.0 ** -22
    live = ~np.isnan(rl)  # [H, T]: rows of a sequence
    rows = live.T[:, :, None] & np.ones(c.D, bool)
    go, gl = host(o), host(lse)
    e3 = es.T[:, :, None]
    tol = (2.0 ** -8 + 2 * e3) * (mag + np.abs(ro)) + (2.0 ** -22 if f32 else 2.0 ** -8) * np.abs(ro) + 1e-30
    with np.errstate(invalid="ignore"):
        err = np.where(rows, np.abs(go - ro), 0.0)
        n = max(1, int(np.max(c.lens)))
        tl = es + (n / 8 + 64) * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(np.isfinite(rl), rl, 0))
        none = np.isneginf(rl)
        el = np.where(none, np.where(np.isneginf(gl), 0.0, np.inf), np.abs(np.where(none, 0, gl) - np.where(none, 0, rl)))
        el = np.where(live, el, 0.0)
    bad = err > np.where(rows, tol, np.inf)
    print(f"[paged attn] {name}: max|dO|={err.max():.3e} ({np.nanmax(err / np.where(rows, tol, 1)):.3f} of the bound) "
          f"max|dLSE|={el.max():.3e} ({(el / tl).max():.3f})", flush=True)
    assert np.isfinite(np.where(rows, go, 0)).all() and not bad.any() and (el <= np.where(live, tl, 1)).all()


# rows, lens, H, heads, D, page: one token to many rows of a key head, lengths around tiles, pages and ranges
CASES = [([1], [1], 1, 1, 64, 16), ([1], [300], 2, 2, 128, 64), ([1, 1], [1000, 31], 12, 12, 128, 32),
         ([1, 1, 1], [1, 33, 700], 16, 2, 64, 16), ([16, 3], [512, 64], 4, 4, 128, 128), ([17], [1999], 3, 3, 64, 256),
         ([5, 0, 2], [255, 40, 257], 12, 4, 128, 16), ([33], [577], 2, 1, 128, 64), ([64], [1100], 3, 3, 128, 64),
         ([65], [65], 2, 2, 64, 16), ([130, 1], [2431, 5], 4, 2, 128, 64), ([300], [1777], 3, 3, 64, 1024),
         ([129], [129], 5, 1, 128, 32), ([520, 1, 77], [1560, 999, 100], 2, 2, 128, 64), ([3], [4100], 40, 1, 128, 64),
         ([1] * 70, list(range(1, 141, 2)), 2, 2, 64, 16), ([257], [600], 10, 2, 64, 128)]


@pytest.mark.parametrize("rows,lens,H,heads,D,page", CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_attention(rows, lens, H, heads, D, page, causal):
    """Everything behind a sequence's places is NaN, in its last page too."""
    c = Case(rows, lens, H, heads, D, page, seed=sum(rows) + D)
    f32 = D == 64
    o, lse = paged().attn_fwd(bf16(c.q), *held(c), causal=causal, out_dtype=torch.float32 if f32 else torch.bfloat16)
    check(f"{(rows[:4], lens[:4], H, heads, D, page, causal)}", o, lse, c, causal, f32=f32)


@pytest.mark.parametrize("rows", [1, 20, 90, 300])
def test_sharp_scores_and_scales(rows):
    """Scores of both signs far apart, a scale of 0 (all places alike) and one of 1."""
    c = Case([rows], [777], 3, 3, 128, 64, seed=rows, sharp=4.0)
    for scale in (0.0, synth.default_scale(128), 1.0):
        o, lse = paged().attn_fwd(bf16(c.q), *held(c), scale=scale, out_dtype=torch.float32)
        check(f"sharp rows={rows} scale={scale:.3f}", o, lse, c, True, scale=scale, f32=True)


@pytest.mark.parametrize("rows", [1, 9, 40, 300])
def test_more_rows_than_places_and_no_places(rows):
    """Tokens before place 0 see nothing; sequences of no places and of no rows."""
    c = Case([rows, rows, 0, rows], [rows // 2, 0, 50, rows + 3], 4, 2, 64, 16, seed=rows)
    for causal in (True, False):
        o, lse = paged().attn_fwd(bf16(c.q), *held(c), causal=causal)
        check(f"rows={rows}", o, lse, c, causal)


@pytest.mark.parametrize("rows,lens", [([1, 1], [500, 3000]), ([200, 30], [500, 3000])])
def test_rows_of_no_sequence_are_left(rows, lens):
    """Rows before the first sequence and behind the last keep what the outputs held, joined ranges or not."""
    c = Case(rows, lens, 2, 2, 128, 64, seed=7, lead=3, tail=4)
    out = torch.full((c.T, 2, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((2, c.T), 7.0, device="cuda")
    paged().attn_fwd(bf16(c.q), *held(c), out=out, lse_out=lse)
    check("left", out, lse, c, True)
    free = torch.ones(c.T, dtype=torch.bool, device="cuda")
    free[3:c.T - 4] = False
    assert bool((out[free] == 5.0).all()) and bool((lse[:, free] == 7.0).all())


@pytest.mark.parametrize("rows", [1, 30, 300])
def test_pages_that_do_not_exist(rows):
    """Entries outside the pool are pages without places, in the middle of a sequence and at its end."""
    c = Case([rows, rows], [900, 700], 4, 2, 128, 32, seed=3)
    c.table[0, 3], c.table[0, 11], c.table[1, 21], c.table[1, 0] = -5, c.k.shape[0], 1 << 30, -(1 << 31)
    for causal in (True, False):
        o, lse = paged().attn_fwd(bf16(c.q), *held(c), causal=causal)
        check(f"holes rows={rows}", o, lse, c, causal)


def test_lens_held_and_hints():
    """Lengths beyond the table and below 0 are held; plans for fewer rows and places than there are."""
    c = Case([4, 4, 4], [896, 512, 500], 2, 2, 64, 64, seed=9)
    cache, table, first, lens = held(c)
    table = table[:, :14].contiguous()
    q = bf16(c.q)
    a = paged().attn_fwd(q, cache, table, first, ints([896, 0, 500]), out_dtype=torch.float32)
    b = paged().attn_fwd(q, cache, table, first, ints([2 ** 31 - 1, -7, 500]), out_dtype=torch.float32)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert bool((a[0][4:8] == 0).all()) and bool(torch.isneginf(a[1][:, 4:8]).all())
    c2 = Case([300, 1], [900, 700], 2, 2, 64, 64, seed=10)
    for hints in ({"max_rows": 1}, {"max_len": 10}, {"max_rows": 1, "max_len": 0}, {"max_rows": 0}):
        o, lse = paged().attn_fwd(bf16(c2.q), *held(c2), **hints)
        check(f"{hints}", o, lse, c2, True)


@pytest.mark.parametrize("rows", [2, 300])
def test_layouts_of_q_o_and_table(rows):
    """q as a slice of a fused projection, head-major q, o within a larger tensor, a table within a wider one."""
    c = Case([rows, rows], [rows + 200, rows + 5], 4, 2, 128, 16, seed=1)
    cache, table, first, lens = held(c)
    q = bf16(c.q)
    ref, lse = paged().attn_fwd(q, cache, table, first, lens)
    wide = torch.randn(c.T, 9, 128, device="cuda").bfloat16()
    wide[:, 2:6] = q
    big = torch.full((c.T + 2, 4, 144), 5.0, dtype=torch.bfloat16, device="cuda")
    tw = torch.full((2, table.shape[1] + 7), 3, dtype=torch.int32, device="cuda")
    tw[:, 4:4 + table.shape[1]] = table
    o, _ = paged().attn_fwd(wide[:, 2:6], cache, tw[:, 4:4 + table.shape[1]], first, lens, out=big[1:-1, :, 8:136],
                            return_lse=False)
    assert torch.equal(o, ref)
    big[1:-1, :, 8:136] = 5.0
    assert bool((big == 5.0).all())
    o, l2 = paged().attn_fwd(q.transpose(0, 1).contiguous().transpose(0, 1), cache, table, first, lens)
    assert torch.equal(o, ref) and torch.equal(l2, lse)


@pytest.mark.parametrize("heads,T", [(2, 1), (5, 3)])
def test_many_key_ranges(heads, T):
    """Few rows against many places: every form of the joining."""
    for n in (300, 600, 1200, 2300, 5000, 17000):
        c = Case([1] * T, [n] + [n // 3] * (T - 1), heads, heads, 64, 64, seed=n)
        o, lse = paged().attn_fwd(bf16(c.q), *held(c), out_dtype=torch.float32)
        check(f"T={T} n={n}", o, lse, c, True, f32=True)


# rows, lens, H, heads, D, page, q_block, count, keep_first, keep_last
SPARSE = [([1], [1], 1, 1, 64, 16, 1, 1, 0, 1), ([1, 1], [500, 2100], 12, 12, 128, 64, 1, 5, 1, 1),
          ([1, 1, 1], [40, 700, 1500], 16, 4, 64, 16, 1, 12, 0, 0), ([70, 5], [900, 333], 4, 2, 128, 32, 16, 6, 1, 2),
          ([200, 0, 65], [200, 100, 1111], 3, 3, 64, 128, 64, 3, 0, 1), ([300], [1300], 8, 2, 128, 64, 64, 7, 2, 2),
          ([50], [640], 6, 1, 128, 16, 128, 9, 3, 3), ([33], [900], 2, 2, 64, 1024, 8, 2, 0, 1),
          ([260], [3000], 2, 1, 128, 64, 7, 4, 1, 0)]


@pytest.mark.parametrize("rows,lens,H,heads,D,page,q_block,count,kf,kl", SPARSE)
@pytest.mark.parametrize("causal", [True, False])
def test_selected_pages(rows, lens, H, heads, D, page, q_block, count, kf, kl, causal):
    """The choice is that of exact scores, and attention sees the chosen pages only."""
    c = Case(rows, lens, H, heads, D, page, seed=sum(lens))
    rng = np.random.default_rng(5)
    mean = synth.normal_bf16(rng, (c.k.shape[0], heads, D), 0.3)
    cache, table, first, n = held(c, bf16(mean))
    q = bf16(c.q)
    got = paged().select_pages(q, cache, table, first, n, count, q_block, kf, kl, causal)
    ref = opaged.select(c.wide()[0], odit.widen(mean), c.table, c.first, c.lens, page, count, q_block, kf, kl, causal)
    assert np.array_equal(got.cpu().numpy(), ref)
    o, lse = paged().attn_pages_fwd(q, cache, table, first, n, got, q_block, causal)
    check(f"selected {(rows, lens, H, heads, D, page, q_block, count)}", o, lse, c, causal, selected=ref, q_block=q_block)


def test_selection_ties_and_nonfinite_scores():
    """Equal scores go to the lower page, NaN counts as -inf, and no infinity displaces the pages always taken."""
    c = Case([1, 1], [40 * 16, 640 * 16], 1, 1, 64, 16, seed=2)
    mean = np.zeros((c.k.shape[0], 1, 64), np.uint16)
    q, k, v = c.wide()
    big = np.uint16(0x7f80)
    for col, bits in ((3, 0x7fc0), (5, int(big)), (8, int(big) | 0x8000), (9, 0x3f80), (12, 0x8000)):
        mean[c.table[1, col], 0, 7] = bits
        mean[c.table[0, col], 0, 7] = bits
    for sign in (1.0, -1.0):
        qs = np.array(c.q)
        qs[:, :, 7] = 0x3f80 if sign > 0 else 0xbf80
        cache, table, first, n = held(c, bf16(mean))
        for count, kf, kl in ((1, 0, 0), (4, 1, 1), (20, 0, 2), (39, 0, 0)):
            got = paged().select_pages(bf16(qs), cache, table, first, n, count, 1, kf, kl)
            ref = opaged.select(odit.widen(qs), odit.widen(mean), c.table, c.first, c.lens, 16, count, 1, kf, kl, True)
            assert np.array_equal(got.cpu().numpy(), ref), (sign, count)


def test_selection_without_queries():
    """No rows, no sequences, no heads of queries: every entry is -1."""
    c = Case([3, 2], [40, 50], 2, 2, 64, 16, seed=1)
    cache, table, first, n = held(c, torch.zeros(c.k.shape[0], 2, 64, dtype=torch.bfloat16, device="cuda"))
    q = bf16(c.q)
    for args in ((q[:0], cache, table, torch.zeros_like(first), n), (q, cache, table[:0], first[:1], n[:0]),
                 (q[:, :0], cache, table, first, n)):
        blocks = args[0].shape[0] // 2 + args[2].shape[0]
        out = torch.full((blocks, 2, 4), 7, dtype=torch.int32, device="cuda")
        paged().select_pages(*args, 4, q_block=2, out=out)
        assert blocks > 0 and bool((out == -1).all())
    for f in (paged().attn_fwd, lambda *a: paged().attn_pages_fwd(*a, torch.zeros(2, 2, 4, dtype=torch.int32, device="cuda"), 2)):
        o, lse = f(q[:0], cache, table, torch.zeros_like(first), n)
        assert o.shape == (0, 2, 64) and lse.shape == (2, 0)


def test_selection_over_many_pages():
    """As many columns as a call takes (131072 bytes of scores in LDS), and scores that differ in their last bits."""
    pages, heads, D = 16384, 1, 64
    rng = np.random.default_rng(0)
    mean = synth.normal_bf16(rng, (64, heads, D))
    # the same 64 pages over and over: hundreds of equal scores of each
    table = (np.arange(pages) % 64).astype(np.int32)[None]
    q = synth.normal_bf16(rng, (1, 1, D))
    cache = paged().PagedCache.zeros(64, 16, heads, D)
    cache = paged().PagedCache(cache.k, cache.v, bf16(mean))
    for n in (pages * 16, pages * 16 - 17):
        for count in (5, 100, 5000):
            got = paged().select_pages(bf16(q), cache, ints(table), ints([0, 1]), ints([n]), count, 1, 2, 3)
            ref = opaged.select(odit.widen(q), odit.widen(mean), table, [0, 1], [n], 16, count, 1, 2, 3, True)
            assert np.array_equal(got.cpu().numpy(), ref), (n, count)


@pytest.mark.parametrize("q_block", [1, 16, 64])
def test_lists_of_any_form(q_block):
    """Lists that no selection gives: unordered, with gaps of -1, indices outside the table, all empty."""
    c = Case([70, 3], [800, 400], 4, 2, 128, 32, seed=4)
    rng = np.random.default_rng(1)
    blocks = c.T // q_block + 2
    lists = np.full((blocks, 2, 9), -1, np.int32)
    for j in range(blocks):
        for h in range(2):
            lists[j, h, :6] = rng.permutation(25)[:6]
            rng.shuffle(lists[j, h])
    lists[1, 0] = -1
    lists[blocks - 1, 1, 2:5] = (1 << 30, -(1 << 31), c.table.shape[1])
    cache, table, first, n = held(c)
    for causal in (True, False):
        o, lse = paged().attn_pages_fwd(bf16(c.q), cache, table, first, n, ints(lists), q_block, causal)
        check(f"lists q_block={q_block}", o, lse, c, causal, selected=lists, q_block=q_block)


@pytest.mark.parametrize("rows,H,heads,D", [(2, 2, 1, 64), (9, 4, 2, 128), (40, 2, 2, 128), (60, 1, 1, 64), (300, 2, 2, 128),
                                            (300, 4, 2, 64)])
@pytest.mark.parametrize("bits", [0x7fc0, 0x7f80, 0xff80])
def test_nonfinite_values_in_places_that_a_query_does_not_see(rows, H, heads, D, bits):
    """An infinity or NaN in the keys or values of a later token of the same chunk is of no account to those before it;
    those from it on get what the definition gives."""
    c = Case([rows, 1], [rows + 700, 90], H, heads, D, 32, seed=rows)
    n, at = rows + 700, rows // 2
    for tensor, place, channel in ((c.v, n - rows + at, 5), (c.v, n - 1, D - 1), (c.k, n - 1 - rows // 4, 3)):
        tensor[c.table[0, place // 32], :, place % 32, channel] = bits
    q, k, v = c.wide()
    with np.errstate(invalid="ignore", over="ignore"):
        ro, rl, _, _ = opaged.attn(q, k, v, c.table, c.first, c.lens, True, synth.default_scale(D))
    o, lse = paged().attn_fwd(bf16(c.q), *held(c), out_dtype=torch.float32)
    go, gl = host(o), host(lse)
    fine, lf = np.isfinite(ro), np.isfinite(rl)
    assert fine[:at].all() and not fine[at:rows].all() and fine[rows:].all()
    # the bounds of `check` where sum p|v| + |O| <= 3 and the largest sum |q||k| scale <= 20 (an infinite key that gives a
    # score of -inf has no part in it): 3 (2^-8 + 2 es), es = 20 * 14 * 2^-24 + 2^-22 < 2^-15; n = 1000
    assert np.isfinite(go[fine]).all() and np.abs(go[fine] - ro[fine]).max() <= 3 * (2.0 ** -8 + 2.0 ** -14)
    assert np.isfinite(gl[lf]).all() and np.abs(gl[lf] - rl[lf]).max() <= 2.0 ** -15 + 189 * 2.0 ** -24 + 2.0 ** -19
    # what is not finite by what the query sees: an infinite value with weight, or NaN
    assert (np.isnan(go) | np.isinf(go))[~fine & np.isnan(ro)].all()
    inf = np.isinf(ro)
    assert np.array_equal(go[inf], ro[inf])


@pytest.mark.parametrize("rows", [20, 200])
def test_nonfinite_values_where_nothing_is_seen(rows):
    """Tokens before place 0 in the same tile as tokens that see an infinity: 0 and -inf."""
    c = Case([rows], [rows // 2], 2, 2, 128, 16, seed=1)
    c.v[c.table[0, 0], :, 0, 7] = 0x7f80
    o, lse = paged().attn_fwd(bf16(c.q), *held(c))
    none = rows - rows // 2
    assert bool((o[:none] == 0).all()) and bool(torch.isneginf(lse[:, :none]).all())
    assert bool(torch.isposinf(o[none:, :, 7]).all()) and bool(torch.isfinite(o[none:, :, :7]).all())


@pytest.mark.parametrize("rows,q_block", [(70, 16), (200, 64), (130, 128)])
def test_nonfinite_values_in_selected_pages(rows, q_block):
    c = Case([rows], [rows + 500], 4, 2, 64, 16, seed=rows)
    place = rows + 500 - rows // 3
    c.v[c.table[0, place // 16], :, place % 16, 2] = 0x7fc0
    clean = Case([rows], [rows + 500], 4, 2, 64, 16, seed=rows)
    pages = -(-(rows + 500) // 16)
    lists = np.tile(np.arange(pages, dtype=np.int32)[::-1], (c.T // q_block + 1, 2, 1))
    o, lse = paged().attn_pages_fwd(bf16(c.q), *held(c), ints(lists), q_block, out_dtype=torch.float32)
    co, cl = paged().attn_pages_fwd(bf16(clean.q), *held(clean), ints(lists), q_block, out_dtype=torch.float32)
    before = place - 500
    assert bool(torch.isfinite(o[:before]).all()) and float((o[:before] - co[:before]).abs().max()) <= 2.0 ** -6
    assert bool(torch.isnan(o[before:, :, 2]).all()) and bool(torch.isfinite(o[before:, :, 3:]).all())
    assert float((lse - cl).abs().max()) <= 2.0 ** -16


def plan(c, q_block=1, count=0, max_rows=None, max_len=None):
    import ctypes
    from paper_2607_28144_amd import _lib
    p = _lib.PagedAttnPlan()
    s = _lib.PagedAttnShape(c.B, c.T, c.H, c.heads, c.D, c.page, q_block, count, c.T if max_rows is None else max_rows,
                            c.table.shape[1] * c.page if max_len is None else max_len)
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    assert _lib.load().regenvc_paged_attn_plan_query(ctypes.byref(s), n_cu, ctypes.byref(p)) == 0
    return p


# rows of each of B sequences, their places (times 1, 2, 3 in turn), H, heads, D, tile rows
TILES = [(2, 5, 700, 2, 2, 128, 16), (2, 30, 700, 2, 2, 64, 32), (70, 60, 200, 4, 4, 64, 64), (40, 60, 260, 4, 4, 128, 64),
         (33, 31, 100, 8, 4, 128, 64), (2, 300, 500, 2, 2, 64, 256)]


@pytest.mark.parametrize("B,rows,places,H,heads,D,tile", TILES)
def test_every_tile(B, rows, places, H, heads, D, tile):
    """Tiles of each number of rows, which the plan says are taken, with sequences that differ."""
    lens = [places * (1 + b % 3) for b in range(B)]
    c = Case([rows - b % 2 for b in range(B)], lens, H, heads, D, 32, seed=tile + D)
    assert plan(c, max_rows=rows).tile_rows == tile
    o, lse = paged().attn_fwd(bf16(c.q), *held(c), max_rows=rows, out_dtype=torch.float32)
    check(f"tile {tile} D={D}", o, lse, c, True, f32=True)


@pytest.mark.parametrize("D", [64, 128])
def test_tiles_of_selected_pages(D):
    """64 rows of many blocks of queries, each with pages of its own."""
    c = Case([1000, 700], [1200, 701], 5, 5, D, 16, seed=D)
    rng = np.random.default_rng(1)
    blocks = c.T // 64 + 2
    lists = np.sort(np.argsort(rng.random((blocks, 5, 44)))[:, :, :20]).astype(np.int32)
    assert plan(c, 64, 20).tile_rows == 64
    o, lse = paged().attn_pages_fwd(bf16(c.q), *held(c), ints(lists), 64, out_dtype=torch.float32)
    check(f"selected, 64 rows, D={D}", o, lse, c, True, selected=lists, q_block=64, f32=True)


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_ranges_of_one_sequence_and_of_several(rows):
    """Keys cut into ranges, which the plan allows: one long sequence alone, and between short ones."""
    for lens in ([9000], [9000, rows, 130 + rows], [5000, 2000 + rows, 700 + rows, rows]):
        c = Case([rows] * len(lens), lens, 2, 1, 64, 128, seed=rows + len(lens))
        assert plan(c).split == 1
        for causal in (True, False):
            o, lse = paged().attn_fwd(bf16(c.q), *held(c), causal=causal, out_dtype=torch.float32)
            check(f"ranges rows={rows} {lens}", o, lse, c, causal, f32=True)
