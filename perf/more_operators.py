"""Operators of a key/value cache in pages, for a block that streams tokens, and the sizes at which a program calls them.

A pool holds keys and values in pages, bf16 [pages, key heads, places of a page, D]; row b of `table` names the pages of
sequence b in order.  New tokens of all sequences stand in one packed [T, heads, D] tensor, those of sequence b in rows
first[b] .. first[b + 1] - 1; they are the last ones of its lens[b] places.

Kinds of case (`"kind"`):
  append  the step before attention in one pass: norm of every head of q and k, rotation by position (neighbouring
          channels or the halves of the rotated part as pairs), keys and values to their places, and with means the
          mean key of each page that they touch (paged.append)
  attn    attention of the new tokens to the places of their sequence, those after them left out (paged.attn_fwd)
  sparse  the pages whose mean key scores best for a block of queries (paged.select_pages), and attention to those
          only (paged.attn_pages_fwd)
"""
import math

import numpy as np
import torch

DEV = "cuda"
EPS = 1e-6
own = False


def listed():
    return [
        # one token of one stream: launch latency
        {"name": "append_token", "kind": "append", "rows": "1", "lens": "10920", "H": 12, "Hkv": 12, "D": 128, "page": 64,
         "norm": True, "layout": "interleaved", "rot": 128, "factor": 1.0, "means": True},
        # a token of each of 64 streams, four query heads to a key head, half of the head rotated, stretched positions
        {"name": "append_streams", "kind": "append", "rows": ",".join(["1"] * 64),
         "lens": ",".join(str(1 + 173 * i) for i in range(64)), "H": 16, "Hkv": 4, "D": 64, "page": 16,
         "norm": False, "layout": "half", "rot": 32, "factor": 4.0, "means": False},
        # a latent frame's tokens of each of seven streams
        {"name": "append_frames", "kind": "append", "rows": ",".join(["1560"] * 7),
         "lens": "1560,1570,1700,2047,2621,3120,4681", "H": 12, "Hkv": 12, "D": 128, "page": 64,
         "norm": True, "layout": "half", "rot": 128, "factor": 1.0, "means": True},
        # one query against three windows
        {"name": "attn_token", "kind": "attn", "rows": "1", "lens": "32760", "H": 12, "Hkv": 12, "D": 128, "page": 64,
         "causal": True},
        # sixteen streams of their own ages, a query each, small pages
        {"name": "attn_streams", "kind": "attn", "rows": ",".join(["1"] * 16),
         "lens": "1,77,300,780,1365,1560,2730,3120,4097,4680,5460,6240,7800,9001,10919,10920", "H": 16, "Hkv": 4, "D": 64,
         "page": 16, "causal": True},
        # chunks of several lengths in one call, five query heads to a key head
        {"name": "attn_ragged", "kind": "attn", "rows": "1365,512,257,77,52,1,1", "lens": "1365,2072,10920,77,4097,9001,3120",
         "H": 20, "Hkv": 4, "D": 128, "page": 128, "causal": True},
        # a latent frame's tokens behind twenty others, all of them visible to one another
        {"name": "attn_frame", "kind": "attn", "rows": "1560", "lens": "32760", "H": 12, "Hkv": 12, "D": 128, "page": 64,
         "causal": False},
        # a whole window from an empty cache
        {"name": "attn_window", "kind": "attn", "rows": "10920", "lens": "10920", "H": 12, "Hkv": 12, "D": 128, "page": 64,
         "causal": True},
        # one query that reads 16 of 512 pages
        {"name": "sparse_token", "kind": "sparse", "rows": "1", "lens": "32760", "H": 12, "Hkv": 12, "D": 128, "page": 64,
         "causal": True, "q_block": 1, "count": 16, "keep_first": 1, "keep_last": 1},
        # sixteen streams of their own ages
        {"name": "sparse_streams", "kind": "sparse", "rows": ",".join(["1"] * 16),
         "lens": "1,300,1365,3120,4680,7800,10919,10920,12480,15600,17160,20280,21840,25001,31200,32760", "H": 16, "Hkv": 4,
         "D": 64, "page": 32, "causal": True, "q_block": 1, "count": 32, "keep_first": 1, "keep_last": 2},
        # a latent frame's tokens behind twenty others, an eighth of the pages for every 64 queries
        {"name": "sparse_frame", "kind": "sparse", "rows": "1560", "lens": "32760", "H": 12, "Hkv": 12, "D": 128, "page": 64,
         "causal": False, "q_block": 64, "count": 64, "keep_first": 1, "keep_last": 25},
        # a whole window from an empty cache, four query heads to a key head
        {"name": "sparse_window", "kind": "sparse", "rows": "10920", "lens": "10920", "H": 16, "Hkv": 4, "D": 128, "page": 64,
         "causal": True, "q_block": 64, "count": 32, "keep_first": 1, "keep_last": 2},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "sparse", "sparse"])
    D, G, Hkv = rng.choice([64, 128]), rng.choice([1, 1, 2, 4, 5]), rng.choice([1, 3, 4, 12])
    page, B = rng.choice([16, 32, 64, 128]), rng.choice([1, 1, 2, 5, 16])
    c = {"kind": kind, "H": G * Hkv, "Hkv": Hkv, "D": D, "page": page}
    if kind == "append":
        rows = [_log(rng, 1, min(10920, 10 ** 7 // (B * (G + 2) * Hkv * D))) for _ in range(B)]
        lens = [n + rng.choice([0, _log(rng, 1, 4680)]) for n in rows]
        layout = rng.choice(["none", "half", "half", "interleaved"])
        c.update(norm=rng.random() < 0.5, layout=layout, rot=rng.choice([D // 4, D // 2, D, D]) if layout != "none" else 0,
                 factor=rng.choice([1.0, 1.0, 4.0, 8.0]), means=rng.random() < 0.5)
    else:
        # many rows or a few; what they read stays below the largest listed case's products and the pool below its own
        most = rng.choice([1, 4, 100, 10920])
        rows = [min(most, _log(rng, 1, 10920)) for _ in range(B)]
        top = 3 * 10 ** 11 // (4 * G * Hkv * D)
        while sum(n * n for n in rows) > top:
            rows = [max(1, n // 2) for n in rows]
        lens = [_log(rng, n, min(32760, top // (B * n), 400000 // (B * Hkv))) for n in rows]
        lens = [max(n, m) for n, m in zip(rows, lens)]
        c.update(causal=rng.random() < 0.7)
        if kind == "sparse":
            first, last = rng.choice([0, 1, 2]), rng.choice([0, 1, 4])
            c.update(q_block=1 if most == 1 else rng.choice([16, 64, 128]), count=max(1, first + last, _log(rng, 1, 96)),
                     keep_first=first, keep_last=last)
    c.update(rows=",".join(map(str, rows)), lens=",".join(map(str, lens)))
    return c


# ---------------------------------------------------------------- inputs
class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def f32(self, *shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=self.g, device=DEV, dtype=torch.float32) * std + mean

    def bf16(self, *shape, std=1.0, mean=0.0):
        return self.f32(*shape, std=std, mean=mean).to(torch.bfloat16)

    def order(self, n):
        return torch.randperm(n, generator=self.g, device=DEV)


def _ints(text):
    return [int(n) for n in text.split(",")]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _turns(case):
    """Turns per position of each rotated pair, in 64 bits; positions stretched by `factor`."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV)
    return 10000.0 ** (-2 * i / case["rot"]) / (2 * math.pi * case["factor"])


def _inputs(case, seed):
    r = _Rand(seed)
    H, Hkv, D, page = (case[n] for n in ("H", "Hkv", "D", "page"))
    rows, lens = _ints(case["rows"]), _ints(case["lens"])
    need = [-(-n // page) for n in lens]
    pages, T = sum(need) + 3, sum(rows)
    # the pool is in use: pages in any order, old tokens' keys in all of them, alike within a page (tokens of one place)
    near = r.f32(pages, Hkv, 1, D, std=0.6)
    d = {"k": (r.f32(pages, Hkv, page, D) + near).to(torch.bfloat16), "v": r.bf16(pages, Hkv, page, D),
         "q": r.bf16(T, H, D), "lens": _i32(lens), "first": _i32([sum(rows[:b]) for b in range(len(rows) + 1)])}
    order = r.order(pages).to(torch.int32)
    d["table"] = torch.zeros(len(rows), max(need), dtype=torch.int32, device=DEV)
    for b, n in enumerate(need):
        d["table"][b, :n] = order[sum(need[:b]):sum(need[:b + 1])]
    if case["kind"] == "append":
        # q, k and v as a fused projection leaves them
        qkv = r.bf16(T, H + 2 * Hkv, D, std=2.0)
        d["q"], d["k_new"], d["v_new"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        if case["norm"]:
            d["w_q"], d["w_k"] = r.bf16(D, std=0.1, mean=1.0), r.bf16(D, std=0.1, mean=1.0)
    if case["kind"] == "sparse" or case.get("means"):
        d["means"] = d["k"].double().mean(2).to(torch.bfloat16)
    return d


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2607_28144_amd import paged
        s["cache"] = paged.PagedCache(s.pop("k"), s.pop("v"), s.pop("means", None))
        if case["kind"] == "append" and case["rot"]:
            s["rotary"] = paged.Rotary(case["rot"], theta=10000.0, layout=case["layout"], scaling="linear", factor=case["factor"],
                                       device=DEV)
    elif case["kind"] == "append" and case["rot"]:
        s["turns"] = _turns(case)
    return s


# ---------------------------------------------------------------- the plain form
def _split(case):
    """Sequences as (b, first row, end row, places)."""
    at = 0
    for b, (n, m) in enumerate(zip(_ints(case["rows"]), _ints(case["lens"]))):
        yield b, at, at + n, m
        at += n


def _norm_rope(x, w, pos, s):
    """x [T, heads, D] float32, normed over D where there are weights and rotated by the positions [T]."""
    case = s["case"]
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    rot = case["rot"]
    if not rot:
        return x
    angle = 2 * math.pi * torch.frac(pos.double()[:, None] * s["turns"])  # [T, rot / 2]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if case["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _places(s):
    """Sequence and place of each new token."""
    first, lens = s["first"].long(), s["lens"].long()
    n = first[1:] - first[:-1]
    seq = torch.repeat_interleave(torch.arange(len(lens), device=DEV), n, output_size=s["q"].shape[0])
    t = torch.arange(s["q"].shape[0], device=DEV)
    return seq, t - first[seq] + (lens - n)[seq]


def _plain_append(s):
    case = s["case"]
    page = case["page"]
    seq, pos = _places(s)
    q = _norm_rope(s["q"].float(), s.get("w_q"), pos, s).to(torch.bfloat16)
    k = _norm_rope(s["k_new"].float(), s.get("w_k"), pos, s).to(torch.bfloat16)
    at = s["table"].long()[seq, pos // page]
    s["k"][at, :, pos % page], s["v"][at, :, pos % page] = k, s["v_new"]
    if "means" not in s:
        return q, s["k"], s["v"]
    # the pages that the new tokens touch, each with as many places as its sequence has there
    touched, back = torch.unique(at, return_inverse=True)
    filled = torch.zeros(len(touched), dtype=torch.long, device=DEV)
    filled.scatter_reduce_(0, back, pos % page + 1, "amax")
    valid = torch.arange(page, device=DEV)[None] < filled[:, None]
    sums = torch.where(valid[:, None, :, None], s["k"][touched].double(), 0.0).sum(2)
    s["means"][touched] = (sums / filled[:, None, None]).to(torch.bfloat16)
    return q, s["k"], s["v"], s["means"]


def _attend(q, k, v, see, scale):
    """q [heads, rows, D], k and v [heads, places, D], float32, see [heads or 1, rows, places]: output, LSE [heads, rows]."""
    z = torch.where(see, torch.matmul(q, k.transpose(1, 2).contiguous()) * scale, -math.inf)
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(m == -math.inf, 0.0, m))
    l = p.sum(-1, keepdim=True)
    o = torch.where(l > 0, torch.matmul(p, v) / torch.where(l > 0, l, 1.0), 0.0)
    return o, (m + torch.log(l))[..., 0]


def _pages_of(s, b, m):
    """Keys and values of the first m places of sequence b, float32 [heads, m, D]."""
    page = s["case"]["page"]
    at = s["table"][b, :-(-m // page)].long()
    return [s[n][at].float().transpose(0, 1).flatten(1, 2)[:, :m].contiguous() for n in ("k", "v")]


def _plain_attention(s, chosen=None):
    """Attention of every sequence's rows; of block j of its queries only to the pages chosen[j] [key heads, count]."""
    case = s["case"]
    H, Hkv, D, page = (case[n] for n in ("H", "Hkv", "D", "page"))
    G, scale = H // Hkv, float(torch.tensor(1.0 / math.sqrt(D), dtype=torch.float32))
    o = torch.empty(s["q"].shape, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(H, s["q"].shape[0], dtype=torch.float32, device=DEV)
    for b, r0, r1, m in _split(case):
        k, v = _pages_of(s, b, m)
        place = torch.arange(m, device=DEV)
        for i in range(r0, r1, 2048):
            rows = torch.arange(i, min(i + 2048, r1), device=DEV)
            n = len(rows)
            q = s["q"][i:i + n].float().view(n, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, n * G, D)
            see = (place[None] <= (m - r1 + rows)[:, None]) if case["causal"] else torch.ones(n, m, dtype=torch.bool, device=DEV)
            see = see[None]
            if chosen is not None:
                block = (rows - r0) // case["q_block"] + r0 // case["q_block"] + b
                picks = chosen[block].long()  # [n, Hkv, count], -1 for none
                mark = torch.zeros(n, Hkv, -(-m // page) + 1, dtype=torch.bool, device=DEV).scatter_(2, picks + 1, True)
                see = see & mark[:, :, 1:].repeat_interleave(page, 2)[..., :m].transpose(0, 1)
            oh, lh = _attend(q, k, v, see.repeat_interleave(G, 1), scale)
            o[i:i + n] = oh.view(Hkv, n, G, D).permute(1, 0, 2, 3).reshape(n, H, D).to(torch.bfloat16)
            lse[:, i:i + n] = lh.view(Hkv, n, G).permute(0, 2, 1).reshape(H, n)
    return o, lse


def _plain_select(s):
    """The pages of each block of queries, in ascending order, -1 behind the last: int32 [blocks, key heads, count]."""
    case = s["case"]
    H, Hkv, D, page, Q, count = (case[n] for n in ("H", "Hkv", "D", "page", "q_block", "count"))
    T, B = s["q"].shape[0], len(s["lens"])
    out = torch.full((T // Q + B, Hkv, count), -1, dtype=torch.int32, device=DEV)
    for b, r0, r1, m in _split(case):
        n = -(-(r1 - r0) // Q)
        end = torch.clamp((torch.arange(n, device=DEV) + 1) * Q, max=r1 - r0) + (m - (r1 - r0)) if case["causal"] \
            else torch.full((n,), m, device=DEV)
        seen = ((end + page - 1) // page)[:, None]  # pages with a place that the block's last query sees
        # the rows' queries summed over a block and the heads that share a key head, in 64 bits
        q = torch.zeros(n * Q, Hkv, D, dtype=torch.float64, device=DEV)
        q[:r1 - r0] = s["q"][r0:r1].double().view(r1 - r0, Hkv, H // Hkv, D).sum(2)
        q = q.view(n, Q, Hkv, D).sum(1).transpose(0, 1).contiguous()
        mean = s["means"][s["table"][b, :-(-m // page)].long()].double()  # [pages, Hkv, D]
        score = torch.matmul(q, mean.permute(1, 2, 0).contiguous()).transpose(0, 1)  # [n, Hkv, pages]
        score = torch.where(torch.isnan(score), -math.inf, score).clamp(max=torch.finfo(torch.float64).max)
        at = torch.arange(mean.shape[0], device=DEV)[None]
        kept = (at < case["keep_first"]) | (at >= seen - case["keep_last"])
        score = torch.where(kept[:, None], math.inf, score)
        score = torch.where((at < seen)[:, None], score, -math.inf)
        best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :count]
        best = torch.where(best < seen[:, None], best, 1 << 30).sort(-1).values
        best = torch.where(best < 1 << 30, best, -1).to(torch.int32)
        j = r0 // Q + b
        out[j:j + n, :, :best.shape[2]] = best
    return out


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    k = case["kind"]
    if not own:
        if k == "append":
            return _plain_append(s)
        if k == "attn":
            return _plain_attention(s)
        chosen = _plain_select(s)
        return (*_plain_attention(s, chosen), chosen)
    from paper_2607_28144_amd import paged
    seqs = (s["cache"], s["table"], s["first"], s["lens"])
    if k == "append":
        q = paged.append(*seqs, s["k_new"], s["v_new"], q=s["q"], w_q=s.get("w_q"), w_k=s.get("w_k"), eps=EPS,
                         rotary=s.get("rotary"))
        c = s["cache"]
        return (q, c.k, c.v, c.means) if case["means"] else (q, c.k, c.v)
    if k == "attn":
        return paged.attn_fwd(s["q"], *seqs, causal=case["causal"])
    chosen = paged.select_pages(s["q"], *seqs, case["count"], q_block=case["q_block"], keep_first=case["keep_first"],
                                keep_last=case["keep_last"], causal=case["causal"])
    return (*paged.attn_pages_fwd(s["q"], *seqs, chosen, q_block=case["q_block"], causal=case["causal"]), chosen)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    H, Hkv, D, page = (case[n] for n in ("H", "Hkv", "D", "page"))
    rows, lens = _ints(case["rows"]), _ints(case["lens"])
    T = sum(rows)
    if case["kind"] == "append":
        touched = sum(-(-m // page) - (m - n) // page for n, m in zip(rows, lens))
        return {"bytes": 4 * T * (H + 2 * Hkv) * D + 2 * Hkv * D * touched * case["means"], "flops": 10 * T * (H + Hkv) * D}
    if case["kind"] == "attn":
        pairs = sum(n * m - (n * (n - 1) // 2 if case["causal"] else 0) for n, m in zip(rows, lens))
        return {"bytes": 4 * T * H * D + 4 * T * H + 4 * sum(lens) * Hkv * D, "flops": 4 * H * D * pairs}
    # every page's mean once; of the places, the chosen ones of a query or all, whichever are fewer
    Q, count = case["q_block"], case["count"]
    pairs = places = scores = blocks = 0
    for n, m in zip(rows, lens):
        blocks += -(-n // Q)
        places += min(m, -(-n // Q) * count * page)
        scores += -(-n // Q) * -(-m // page)
        pairs += sum(min(m - (n - i if case["causal"] else 0), count * page) * min(Q, n - i) for i in range(0, n, Q))
    means = 2 * Hkv * D * sum(-(-m // page) for m in lens)
    return {"bytes": 4 * T * H * D + 4 * T * H + 4 * places * Hkv * D + means + 4 * blocks * Hkv * count,
            "flops": 4 * H * D * pairs + 2 * Hkv * D * scores}


# ---------------------------------------------------------------- the same in 64 bits
def _exact_append(s, case):
    H, Hkv, D, page, rot = (case[n] for n in ("H", "Hkv", "D", "page", "rot"))
    keys, values = s["k"].double(), s["v"].double()
    q_out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    marks = []
    for b, r0, r1, m in _split(case):
        start = m - (r1 - r0)
        pos = torch.arange(start, m, device=DEV)
        out = []
        for x, w in ((s["q"][r0:r1].double(), s.get("w_q")), (s["k_new"][r0:r1].double(), s.get("w_k"))):
            if w is not None:
                x = x / torch.sqrt((x * x).sum(2, keepdim=True) / D + EPS) * w.double()
            y = x.clone()
            for i in range(rot // 2):
                i0, i1 = (i, i + rot // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
                a = pos.double() * (math.pow(10000.0, -2.0 * i / rot) / case["factor"])
                c, z = torch.cos(a)[:, None], torch.sin(a)[:, None]
                y[..., i0], y[..., i1] = x[..., i0] * c - x[..., i1] * z, x[..., i0] * z + x[..., i1] * c
            out.append(y)
        q_out[r0:r1] = out[0]
        for p in range(start // page, -(-m // page)):
            lo, hi, at = max(start, p * page), min(m, (p + 1) * page), int(s["table"][b, p])
            keys[at, :, lo - p * page:hi - p * page] = out[1][lo - start:hi - start].transpose(0, 1)
            values[at, :, lo - p * page:hi - p * page] = s["v_new"][r0 + lo - start:r0 + hi - start].double().transpose(0, 1)
            marks.append((at, hi - p * page))
    if not case["means"]:
        return q_out, keys, values
    means = s["means"].double()
    for at, n in marks:
        means[at] = keys[at, :, :n].to(torch.bfloat16).double().sum(1) / n
    return q_out, keys, values, means


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "append":
        return _exact_append(s, case)
    H, Hkv, D, page = (case[n] for n in ("H", "Hkv", "D", "page"))
    G, T, sparse = H // Hkv, s["q"].shape[0], case["kind"] == "sparse"
    Q = case["q_block"] if sparse else 1024
    o = torch.zeros((T, H, D), dtype=torch.float64, device=DEV)
    lse = torch.full((H, T), -math.inf, dtype=torch.float64, device=DEV)
    chosen = torch.full((T // Q + len(s["lens"]), Hkv, case["count"]), -1, dtype=torch.int32) if sparse else None
    scale = float(torch.tensor(1.0 / math.sqrt(D), dtype=torch.float32))
    for b, r0, r1, m in _split(case):
        at = s["table"][b, :-(-m // page)].long()
        for h in range(Hkv):
            k = s["k"][at, h].double().reshape(-1, D)[:m]
            v = s["v"][at, h].double().reshape(-1, D)[:m].contiguous()
            if sparse:
                q = s["q"][r0:r1, h * G:(h + 1) * G].double().sum(1)
                q = torch.stack([c.sum(0) for c in q.split(Q)])
                score = torch.mm(q, s["means"][at, h].double().t().contiguous()).cpu().numpy()
            for j, i in enumerate(range(r0, r1, Q)):
                n = min(Q, r1 - i)
                place = torch.arange(m, device=DEV)
                if sparse:
                    seen = -(-(m - r1 + i + n if case["causal"] else m) // page)
                    must = [p for p in range(seen) if p < case["keep_first"] or p >= seen - case["keep_last"]]
                    order = np.argsort(-score[j, :seen], kind="stable")
                    rest = order[~np.isin(order, must)][:max(0, case["count"] - len(must))]
                    picks = sorted(must + rest.tolist())
                    chosen[r0 // Q + b + j, h, :len(picks)] = torch.tensor(picks, dtype=torch.int32)
                    p = torch.tensor(picks, device=DEV)
                    place = (p[:, None] * page + torch.arange(page, device=DEV)).flatten()
                    place = place[place < m]
                q = s["q"][i:i + n, h * G:(h + 1) * G].double().reshape(n * G, D)
                z = torch.mm(q, k[place].t().contiguous()) * scale
                if case["causal"]:
                    pos = (m - r1 + i + torch.arange(n, device=DEV)).repeat_interleave(G)
                    z = z.masked_fill(place[None] > pos[:, None], -math.inf)
                # a query that none of its block's pages lets see a place has no weight at all
                l = torch.logsumexp(z, 1)
                w = torch.exp(z - torch.where(l == -math.inf, 0.0, l)[:, None])
                o[i:i + n, h * G:(h + 1) * G] = torch.mm(w, v[place]).view(n, G, D)
                lse[h * G:(h + 1) * G, i:i + n] = l.view(n, G).t()
    return (o, lse, chosen.to(DEV)) if sparse else (o, lse)
