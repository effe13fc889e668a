"""The operators of the paged cache together, as a program that streams uses them:
append, choice of pages and attention, step after step, eager and captured, on
streams of their own; long offsets and many sequences."""
import copy

import numpy as np
import pytest

from oracle import dit as odit
from oracle import paged as opaged
from paged_cases import Case
from paper_2607_28144_amd import synth
from test_gpu_paged import bf16, check, held, host, ints, paged, plan

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


class Stream:
    """Sequences that grow: pages are taken from the pool as they are needed, in any order."""

    def __init__(self, B, H, heads, D, page, pages, seed):
        rng = np.random.default_rng(seed)
        self.B, self.H, self.heads, self.D, self.page, self.rng = B, H, heads, D, page, rng
        old = [synth.normal_bf16(rng, s) for s in ((pages, heads, page, D),) * 2 + ((pages, heads, D),)]
        self.cache = paged().PagedCache(*(bf16(x) for x in old))
        self.k, self.v, self.means = (odit.widen(x) for x in old)
        self.free = list(rng.permutation(pages))
        self.table = np.full((B, pages // B), -1, np.int32)
        self.lens = np.zeros(B, np.int32)
        self.w = [synth.normal_bf16(rng, (D,)) for _ in range(2)]
        self.rotary = paged().Rotary(D, layout="half", scaling="parts", factor=4.0, original_len=64)

    def grow(self, rows):
        self.lens = (self.lens + rows).astype(np.int32)
        for b in range(self.B):
            for c in range(-(-int(self.lens[b]) // self.page)):
                if self.table[b, c] < 0:
                    self.table[b, c] = self.free.pop()
        return np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)


def test_steps_of_a_stream():
    """Chunks, single tokens and sequences without new tokens in turn.  q, keys, means and the choice are compared with the
    oracle on the keys as the cache holds them, so that a rounding does not decide which pages are right."""
    s = Stream(3, 4, 2, 64, 16, 60, 1)
    q_block, count = 16, 6
    for rows in ([40, 3, 0], [1, 1, 1], [1, 1, 1], [0, 70, 33], [130, 1, 1], [1, 1, 0]):
        first = s.grow(rows)
        T = int(first[-1])
        qkv = synth.normal_bf16(s.rng, (T, s.H + 2 * s.heads, s.D), 2.0)
        t = bf16(qkv)
        table, f, n = ints(s.table), ints(first), ints(s.lens)
        q = paged().append(s.cache, table, f, n, t[:, s.H:s.H + s.heads], t[:, s.H + s.heads:], q=t[:, :s.H], w_q=bf16(s.w[0]),
                           w_k=bf16(s.w[1]), rotary=s.rotary)
        x = odit.widen(qkv)
        turns = s.rotary.turns.cpu().numpy()
        rq, rk, s.v, at = opaged.append(x[:, :s.H], x[:, s.H:s.H + s.heads], x[:, s.H + s.heads:], s.k, s.v, s.table, first,
                                        s.lens, odit.widen(s.w[0]), odit.widen(s.w[1]), 1e-6, turns, "half", s.rotary.amplitude)
        gk = host(s.cache.k)
        assert np.array_equal(np.where(at[:, None, :, None], 0, gk), np.where(at[:, None, :, None], 0, s.k))
        for got, ref in ((host(q), rq), (np.where(at[:, None, :, None], gk, 0), np.where(at[:, None, :, None], rk, 0))):
            # a rounding to bf16, and 2e-6 + 24 roundings of the rotated pair, which is no longer than the head's largest
            assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 4e-6 * 2 * np.abs(ref).max(-1, keepdims=True)).all()
        s.k = gk
        assert np.array_equal(host(s.cache.v), s.v)
        s.means = odit.round_bf16(opaged.means(s.k, s.table, first, s.lens, s.means))
        assert np.array_equal(host(s.cache.means), s.means)

        c = Case.__new__(Case)
        c.table, c.first, c.lens, c.D = s.table, first, s.lens, s.D
        c.wide = lambda: (host(q), s.k, s.v)
        o, lse = paged().attn_fwd(q, s.cache, table, f, n, out_dtype=torch.float32)
        check(f"step {rows}", o, lse, c, True, f32=True)
        chosen = paged().select_pages(q, s.cache, table, f, n, count, q_block, 1, 2)
        ref = opaged.select(host(q), s.means, s.table, first, s.lens, s.page, count, q_block, 1, 2, True)
        assert np.array_equal(chosen.cpu().numpy(), ref)
        o, lse = paged().attn_pages_fwd(q, s.cache, table, f, n, chosen, q_block, out_dtype=torch.float32)
        check(f"step {rows}, selected", o, lse, c, True, selected=ref, q_block=q_block, f32=True)


def step(cache, table, first, lens, qkv, H, heads, w, rotary, q_block, count):
    q = paged().append(cache, table, first, lens, qkv[:, H:H + heads], qkv[:, H + heads:], q=qkv[:, :H], w_q=w, w_k=w, rotary=rotary)
    dense = paged().attn_fwd(q, cache, table, first, lens)
    chosen = paged().select_pages(q, cache, table, first, lens, count, q_block, 1, 1)
    return (q, *dense, chosen, *paged().attn_pages_fwd(q, cache, table, first, lens, chosen, q_block))


@pytest.mark.parametrize("rows,q_block", [([1, 1], 1), ([60, 20], 16), ([200, 56], 64)])
def test_captured_steps(rows, q_block):
    """Two graphs of steps on two caches, replayed in turn as their sequences grow (lengths live on the device), with eager
    steps on a third cache between: every replay gives what the eager step gives."""
    B, H, heads, D, page, pages = 2, 4, 2, 128, 32, 64
    rng = np.random.default_rng(2)
    old = [synth.normal_bf16(rng, (pages, heads, page, D)) for _ in range(2)] + [synth.normal_bf16(rng, (pages, heads, D))]
    caches = [paged().PagedCache(*(bf16(x) for x in old)) for _ in range(4)]
    table = ints(rng.permutation(pages).reshape(B, -1))
    T = sum(rows)
    first = ints(np.concatenate([[0], np.cumsum(rows)]))
    w, rotary = bf16(synth.normal_bf16(rng, (D,))), paged().Rotary(D)
    qkv = [torch.zeros(T, H + 2 * heads, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lens = [ints(rows) for _ in range(2)]
    args = lambda i: (table, first, lens[i], qkv[i], H, heads, w, rotary, q_block, 5)  # noqa: E731
    step(caches[3], *args(0))
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(caches[i], *args(i)))
        graphs.append(g)
    eager = [paged().PagedCache(*(bf16(x) for x in old)) for _ in range(2)]
    for i in range(2):
        for part, x in zip((caches[i].k, caches[i].v, caches[i].means), old):
            part.copy_(bf16(x))
    for t in range(3):
        for i in range(2):
            qkv[i].copy_(bf16(synth.normal_bf16(rng, qkv[i].shape)))
            lens[i].copy_(ints(np.array(rows) * (t + 1) + 37 * i))
        for g in graphs:
            g.replay()
        for i in range(2):
            ref = step(eager[i], *args(i))
            torch.cuda.synchronize()
            for got, want in zip(outs[i], ref):
                assert torch.equal(got, want)
            assert torch.equal(caches[i].k, eager[i].k) and torch.equal(caches[i].means, eager[i].means)


def test_streams_of_their_own():
    """Two steps at once on two streams, neither the default one, give what one after the other does."""
    B, H, heads, D, page, pages = 2, 4, 2, 64, 16, 128
    rng = np.random.default_rng(4)
    old = [synth.normal_bf16(rng, (pages, heads, page, D)) for _ in range(2)] + [synth.normal_bf16(rng, (pages, heads, D))]
    table, first, lens = ints(rng.permutation(pages).reshape(B, -1)), ints([0, 150, 151]), ints([900, 1000])
    w, rotary = bf16(synth.normal_bf16(rng, (D,))), paged().Rotary(D, layout="interleaved")
    qkv = [bf16(synth.normal_bf16(rng, (151, H + 2 * heads, D))) for _ in range(2)]
    caches = [paged().PagedCache(*(bf16(x) for x in old)) for _ in range(4)]
    args = lambda i: (table, first, lens, qkv[i % 2], H, heads, w, rotary, 64, 9)  # noqa: E731
    ref = [step(caches[i], *args(i)) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            got.append([step(caches[2 + i], *args(i)) for _ in range(3)][-1])
    torch.cuda.synchronize()
    for i in range(2):
        for a, b in zip(got[i], ref[i]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_offsets_past_32_bits(rows):
    """A pool of more than 2^31 elements, its last pages in use; a table of far more columns than there are pages."""
    page, D, heads = 1024, 128, 2
    pages = (1 << 31) // (heads * page * D) + 9
    c = Case([rows], [2500], 4, heads, D, page, seed=3, spare=0)
    k, v = (torch.empty(pages, heads, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    means = torch.zeros(pages, heads, D, dtype=torch.bfloat16, device="cuda")
    base = pages - c.k.shape[0]
    k[base:], v[base:] = bf16(c.k), bf16(c.v)
    cache = paged().PagedCache(k, v, means)
    table = np.full((1, 200000), -1, np.int32)
    table[0, :c.table.shape[1]] = np.where(c.table[0] >= 0, c.table[0] + base, -1)
    args = (cache, ints(table), ints(c.first), ints(c.lens))
    o, lse = paged().attn_fwd(bf16(c.q), *args)
    check(f"far pages rows={rows}", o, lse, c, True)
    new = bf16(synth.normal_bf16(np.random.default_rng(1), (rows, heads, D)))
    paged().append(*args, new, new)
    for i in (0, rows - 1):
        place = 2500 - rows + i
        assert torch.equal(k[base + c.table[0, place // page], :, place % page], new[i])


def test_more_sequences_than_a_plan_goes_over():
    """Beyond 256 sequences keys are not cut; lengths of 0 to 300, every third sequence without new tokens."""
    B = 1100
    rows = [0 if b % 3 == 2 else 1 + b % 2 for b in range(B)]
    c = Case(rows, [(7 * b) % 300 for b in range(B)], 1, 1, 64, 16, seed=6)
    o, lse = paged().attn_fwd(bf16(c.q), *held(c), out_dtype=torch.float32)
    check("1100 sequences", o, lse, c, True, f32=True)


@pytest.mark.parametrize("B", [65, 200, 256])
def test_sequences_beyond_64(B):
    """More sequences than a wave has lanes, whose keys may be cut: one long one among short ones, some without rows."""
    rows = [0 if b % 7 == 3 else 1 + b % 3 for b in range(B)]
    lens = [4000 if b == B - 2 else 3 + (11 * b) % 200 for b in range(B)]
    c = Case(rows, lens, 2, 1, 64, 64, seed=B)
    assert plan(c).split == 1
    for causal in (True, False):
        o, lse = paged().attn_fwd(bf16(c.q), *held(c), causal=causal, out_dtype=torch.float32)
        check(f"{B} sequences", o, lse, c, causal, f32=True)


def some_heads(c, heads):
    """The case of these key heads alone, for as many query heads."""
    d = copy.copy(c)
    d.q, d.k, d.v, d.H, d.heads = c.q[:, heads], c.k[:, heads], c.v[:, heads], len(heads), len(heads)
    return d


@pytest.mark.parametrize("lead,tail,lens", [(0, 0, 1300), (3, 9, 1300), (120, 0, 1290), (0, 30, 170)])
def test_one_sequence_of_more_tiles_than_compute_units(lead, tail, lens):
    """Whole tiles for one round of workgroups and ranges of the others' keys, with rows of no sequence and few places."""
    rows, count, page, heads = 168 - lead - tail, 64, 16, [0, 9, 17, 25]
    c = Case([rows], [lens], 26, 26, 64, page, seed=lead + tail, lead=lead, tail=tail)
    c.table = np.pad(c.table, ((0, 0), (0, 83 - c.table.shape[1])), constant_values=-1)
    p = plan(c, 16, count, max_len=1300)
    assert p.split == 1 and p.tile_rows == 16
    blocks = c.T // 16 + 1
    lists = np.sort(np.argsort(np.random.default_rng(lens).random((blocks, 26, 82)))[:, :, :count]).astype(np.int32)
    lists[::3, :, 50:] = -1
    o = torch.full((c.T, 26, 64), 7.0, device="cuda")
    lse = torch.full((26, c.T), 7.0, device="cuda")
    for causal in (True, False):
        paged().attn_pages_fwd(bf16(c.q), *held(c), ints(lists), 16, causal=causal, max_len=1300, out_dtype=torch.float32,
                               out=o, lse_out=lse)
        check(f"round and rest {lead} {tail}", o[:, heads], lse[heads], some_heads(c, heads), causal, selected=lists[:, heads],
              q_block=16, f32=True)
        assert bool((o[:lead] == 7).all()) and bool((o[c.T - tail:] == 7).all())
        assert bool((lse[:, :lead] == 7).all()) and bool((lse[:, c.T - tail:] == 7).all())


@pytest.mark.parametrize("rows", [257, 320, 200])
def test_one_sequence_of_more_large_tiles_than_compute_units(rows):
    """The same of 256 rows: planned for 320 tokens of 130 heads."""
    heads = [0, 1, 64, 129]
    c = Case([rows], [2100], 130, 130, 64, 64, seed=rows, tail=320 - rows)
    assert plan(c).split == 1 and plan(c).tile_rows == 256
    for causal in (True, False):
        o, lse = paged().attn_fwd(bf16(c.q), *held(c), causal=causal, out_dtype=torch.float32)
        check(f"large round and rest {rows}", o[:, heads], lse[heads], some_heads(c, heads), causal, f32=True)


@pytest.mark.parametrize("causal", [True, False])
def test_a_whole_window_of_more_large_tiles_than_compute_units(causal):
    """600 of 2100 places are new: a causal call keeps its tiles whole, one that sees them all does not."""
    heads = [0, 3, 89]
    c = Case([600], [2100], 90, 90, 64, 64, seed=9)
    need = paged()._need((1, 600, 90, 90, 64, 64, 1, 0, 600, c.table.shape[1] * 64, int(causal)), 0)
    assert (need > 0) == (not causal)
    o, lse = paged().attn_fwd(bf16(c.q), *held(c), causal=causal, out_dtype=torch.float32)
    check(f"window causal={causal}", o[:, heads], lse[heads], some_heads(c, heads), causal, f32=True)
