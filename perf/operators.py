"""Operators of a block that streams video in four bits, and the sizes at which a program calls them.

Kinds of case (`"kind"`):
  linear  a linear layer with weights in MXFP4 (blocks of 32 values of 4 bits under a power-of-two scale): the bf16
          activations are brought to MXFP4 as well and multiplied, with bias or with bias and GELU (mx.linear_fwd)
  cache   attention of the queries to a key/value cache held in MXFP4, a length per sequence (mx.attn_cache_fwd); with
          append the step before it too: the new tokens' keys and values go to the cache from `start` on, wrapping at
          its end (mx.KvCache.append), and the cache's values come back (mx.KvCache.values)
  norm    the seam between two branches: x' = alpha x + gate N_post(y), h = N_pre(x') (1 + scale) + shift, or with
          bf16 weights in place of the modulation (dit.residual_norm_fwd)
  grad    the gradients of that seam (dit.residual_norm_bwd)
"""
import math

import torch

DEV = "cuda"
EPS = 1e-6
own = False


def listed():
    return [
        # the conditioning vector of one denoising step through a linear layer: launch latency, weights read once
        {"name": "linear_one_row", "kind": "linear", "M": 1, "N": 1536, "K": 1536, "gelu": False},
        # a few streams' vectors through the widest layer
        {"name": "linear_few_rows", "kind": "linear", "M": 21, "N": 8960, "K": 1536, "gelu": True},
        # one GPU's tokens of eight, down projection
        {"name": "linear_shard", "kind": "linear", "M": 1365, "N": 1536, "K": 8960, "gelu": False},
        # a window's tokens, up projection
        {"name": "linear_window", "kind": "linear", "M": 10920, "N": 8960, "K": 1536, "gelu": True},
        # one query against a window in the cache
        {"name": "cache_token", "kind": "cache", "B": 1, "S": 1, "H": 12, "Hkv": 12, "D": 128, "cap": 10920,
         "lens": "10920", "append": False},
        # sixteen streams of their own ages, four query heads to a key head
        {"name": "cache_streams", "kind": "cache", "B": 16, "S": 3, "H": 16, "Hkv": 4, "D": 64, "cap": 10920,
         "lens": "1,77,300,780,1365,1560,2730,3120,4097,4680,5460,6240,7800,9001,10919,10920",
         "append": False},
        # a strip of new tokens joins a rolling cache of two latent frames and attends to it
        {"name": "cache_step", "kind": "cache", "B": 2, "S": 52, "H": 12, "Hkv": 12, "D": 128, "cap": 3120,
         "lens": "3120,1612", "append": True},
        # a latent frame's tokens against three windows in the cache
        {"name": "cache_frame", "kind": "cache", "B": 1, "S": 1560, "H": 12, "Hkv": 12, "D": 128, "cap": 32760,
         "lens": "32760", "append": False},
        # a single row
        {"name": "norm_row", "kind": "norm", "rows": 1, "C": 1536, "norm": "layer", "post": "none", "group": 0, "mod": True},
        # a window's tokens, a modulation per latent frame, norms on both sides of the branch
        {"name": "norm_window", "kind": "norm", "rows": 10920, "C": 1536, "norm": "layer", "post": "rms", "group": 1560,
         "mod": True},
        # training on one latent frame, norms with weights only
        {"name": "grad_frame", "kind": "grad", "rows": 1560, "C": 2048, "norm": "rms", "post": "rms", "group": 0, "mod": False},
        # training on a window, a modulation per latent frame
        {"name": "grad_window", "kind": "grad", "rows": 10920, "C": 1536, "norm": "layer", "post": "none", "group": 1560,
         "mod": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "cache", "cache", "norm", "grad"])
    if kind == "linear":
        M, N = _log(rng, 1, 10920), 16 * _log(rng, 8, 560)
        K = 8 * _log(rng, 16, min(1120, 10920 * 8960 * 192 // (M * N)))
        return {"kind": kind, "M": M, "N": N, "K": K, "gelu": rng.random() < 0.5}
    if kind == "cache":
        D, G = rng.choice([64, 128]), rng.choice([1, 1, 2, 4, 5])
        B, Hkv, S = rng.choice([1, 1, 2, 5, 16]), rng.choice([1, 3, 4, 12]), _log(rng, 1, 1560)
        S = min(S, max(1, 5 * 10 ** 7 // (B * Hkv * G * D)))
        append = S <= 100 and rng.random() < 0.4
        top = 1560 * 32760 * 12 * 128 // (B * S * Hkv * G * D)
        cap = _log(rng, 256, max(257, min(4000 if append else 32760, top, 393216 // (B * Hkv))))
        lens = [min(cap, max(1, _log(rng, 1, 3 * cap))) for _ in range(B)]
        return {"kind": kind, "B": B, "S": S, "H": Hkv * G, "Hkv": Hkv, "D": D, "cap": cap,
                "lens": ",".join(str(max(n, min(S, cap)) if append else n) for n in lens), "append": append}
    rows = _log(rng, 1, 10920)
    C = 8 * _log(rng, 32, 512)
    while rows * C > 10920 * 1536:
        rows = rows * 3 // 4
    return {"kind": kind, "rows": rows, "C": C, "norm": rng.choice(["layer", "rms"]),
            "post": rng.choice(["none", "rms", "layer"]), "group": rng.choice([0, 0, 300, max(1, rows // 3)]),
            "mod": rng.random() < 0.6}


# ---------------------------------------------------------------- inputs
class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def f32(self, *shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=self.g, device=DEV, dtype=torch.float32) * std + mean

    def bf16(self, *shape, std=1.0, mean=0.0):
        return self.f32(*shape, std=std, mean=mean).to(torch.bfloat16)


def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def _post(case):
    return None if case["post"] == "none" else case["post"]


def _groups(case):
    return -(-case["rows"] // case["group"]) if case["group"] else 1


def _inputs(case, seed):
    r = _Rand(seed)
    k = case["kind"]
    if k == "linear":
        # normalized and modulated activations: some channels an order of magnitude above the rest
        M, N, K = case["M"], case["N"], case["K"]
        return {"a": (r.f32(M, K) * (1 + 0.5 * r.f32(K)) * torch.exp(0.7 * r.f32(K))).to(torch.bfloat16),
                "w": r.bf16(N, K, std=0.02), "b": r.bf16(N, std=0.02)}
    if k == "cache":
        B, S, H, Hkv, D, cap = (case[n] for n in ("B", "S", "H", "Hkv", "D", "cap"))
        d = {"q": r.bf16(B, S, H, D), "k": r.bf16(B, cap, Hkv, D), "v": r.bf16(B, cap, Hkv, D),
             "lens": torch.tensor(_lens(case), dtype=torch.int32, device=DEV)}
        if case["append"]:
            # a sequence whose cache is full has been through it once: its new tokens take the oldest ones' places
            d["start"] = torch.tensor([n - min(S, cap) if n < cap else cap + n // 2 for n in _lens(case)], dtype=torch.int32,
                                      device=DEV)
            d["k_new"], d["v_new"] = r.bf16(B, S, Hkv, D), r.bf16(B, S, Hkv, D)
        return d
    rows, C, G = case["rows"], case["C"], _groups(case)
    d = {"x": r.f32(rows, C, std=2.0) * torch.exp(0.5 * r.f32(C)), "y": r.bf16(rows, C), "gate": r.f32(G, C, std=0.5)}
    if case["mod"]:
        d["scale"], d["shift"] = r.f32(G, C, std=0.5), r.f32(G, C, std=0.5)
    else:
        d["w"] = r.bf16(C, std=0.1, mean=1.0)
        if case["norm"] == "layer":
            d["b"] = r.bf16(C, std=0.1)
    if _post(case):
        d["post_w"] = r.bf16(C, std=0.1, mean=1.0)
    if k == "grad":
        d["gh"], d["gx"] = r.bf16(rows, C), r.f32(rows, C)
    return d


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "linear":
        # the weights are quantised when the model is loaded
        if own:
            from paper_2607_28144_amd import mx
            s["w"] = mx.quantize(s["w"])
        else:
            s["w"] = _quantize(s["w"])
    if case["kind"] == "cache":
        # keys and values that earlier steps left in the cache, in places behind the lengths too
        k, v = s.pop("k"), s.pop("v")
        if own:
            from paper_2607_28144_amd import mx
            s["cache"] = mx.KvCache(case["B"], case["cap"], case["Hkv"], case["D"], device=DEV)
            s["cache"].append(k, v, torch.zeros(case["B"], dtype=torch.int32, device=DEV))
        else:
            s["k"], s["v"] = _quantize(k), _quantize(v)
    return s


# ---------------------------------------------------------------- the plain form
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantize(x):
    """MXFP4 of x [..., n] along its last axis: codes [..., blocks, 32] (sign and magnitude index) and the exponents of
    the blocks' scales [..., blocks, 1]; the last block is filled up with zeros.  A block's scale is two to the
    (exponent of its largest magnitude - 2); values are rounded to nearest, ties to the even code, and held at 6."""
    x = x.float()
    n = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -n % 32)).unflatten(-1, (-1, 32))
    e = torch.frexp(x.abs().amax(-1, keepdim=True))[1]
    e = torch.where((x == 0).all(-1, keepdim=True), -127, torch.clamp(e - 3, -127, 127)).to(torch.int16)
    v = torch.ldexp(x, -e.to(torch.int32))
    a = v.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8) + (a >= 1.75).to(torch.uint8)
            + (a > 2.5).to(torch.uint8) + (a >= 3.5).to(torch.uint8) + (a > 5.0).to(torch.uint8))
    return code + 8 * (v < 0).to(torch.uint8), e, n


def _values(q, lo=None, hi=None):
    """The float32 values that codes and scales stand for (of one range of the leading axis)."""
    code, e, n = q
    if lo is not None:
        code, e = code[lo:hi], e[lo:hi]
    grid = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), dtype=torch.float32, device=code.device)
    return torch.ldexp(grid[code.int()], e.to(torch.int32)).flatten(-2)[..., :n]


def _attend(q, k, v, n, scale):
    """q [S, G, D], k and v [cap, D] of one key head, float32, n valid places: output [S, G, D] and LSE [G, S]."""
    S, G, D = q.shape
    valid = torch.arange(k.shape[0], device=q.device) < n
    v = torch.where(valid[:, None], v, 0.0)
    kt = torch.where(valid[:, None], k, 0.0).t().contiguous()
    rows = q.reshape(S * G, D)
    out, lse = torch.empty_like(rows), torch.empty(S * G, dtype=rows.dtype, device=q.device)
    for i in range(0, S * G, 8192):
        s = torch.where(valid[None, :], torch.mm(rows[i:i + 8192], kt) * scale, -math.inf)
        m = s.amax(1, keepdim=True)
        m0 = torch.where(m == -math.inf, 0.0, m)
        p = torch.exp(s - m0)
        l = p.sum(1, keepdim=True)
        out[i:i + 8192] = torch.where(l > 0, torch.mm(p, v) / torch.where(l > 0, l, 1.0), 0.0)
        lse[i:i + 8192] = (m + torch.log(l))[:, 0]
    return out.view(S, G, D), lse.view(S, G).t()


def _norm32(x, kind):
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    return x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)


def _per_row(t, case):
    """A [groups, C] vector set as one row per row of the batch."""
    if t.shape[0] == 1:
        return t
    return t[torch.arange(case["rows"], device=t.device) // case["group"]]


def _column_sums(t, case):
    """Sums of t [rows, C] over each group's rows: [groups, C]."""
    if not case["group"]:
        return t.sum(0, keepdim=True)
    return torch.stack([c.sum(0) for c in t.split(case["group"])])


def _plain(s):
    case = s["case"]
    k = case["kind"]
    if k == "linear":
        a = _values(_quantize(s["a"]))
        y = torch.mm(a, _values(s["w"]).t()) + s["b"].float()
        if case["gelu"]:
            y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
        return y.to(torch.bfloat16)
    if k == "cache":
        B, S, H, Hkv, D, cap = (case[n] for n in ("B", "S", "H", "Hkv", "D", "cap"))
        if case["append"]:
            for old, new in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
                code, e, _ = _quantize(new[:, max(0, S - cap):])
                at = (s["start"][:, None].long() + torch.arange(max(0, S - cap), S, device=DEV)) % cap
                b = torch.arange(B, device=DEV)[:, None].expand_as(at)
                old[0][b, at], old[1][b, at] = code, e
        scale = float(torch.tensor(1.0 / math.sqrt(D), dtype=torch.float32))
        o = torch.empty((B, S, H, D), dtype=torch.bfloat16, device=DEV)
        lse = torch.empty((B, H, S), dtype=torch.float32, device=DEV)
        G = H // Hkv
        for b in range(B):
            kb, vb = _values(s["k"], b, b + 1)[0], _values(s["v"], b, b + 1)[0]
            for h in range(Hkv):
                oh, lh = _attend(s["q"][b, :, h * G:(h + 1) * G].float(), kb[:, h], vb[:, h], s["lens"][b], scale)
                o[b, :, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G] = oh.to(torch.bfloat16), lh
        if case["append"]:
            return o, lse, _values(s["k"]).to(torch.bfloat16), _values(s["v"]).to(torch.bfloat16)
        return o, lse
    gate, y = _per_row(s["gate"], case), s["y"].float()
    w = s["post_w"].float() if _post(case) else None
    n_post = _norm32(y, case["post"]) if _post(case) else y
    u = n_post * w if _post(case) else y
    mul = 1 + _per_row(s["scale"], case) if case["mod"] else s["w"].float()
    if k == "norm":
        x = s["x"] + gate * u
        h = _norm32(x, case["norm"]) * mul
        if case["mod"]:
            h = h + _per_row(s["shift"], case)
        elif case["norm"] == "layer":
            h = h + s["b"].float()
        return x, h.to(torch.bfloat16)

    def back(x, n, g, kind):
        """Gradient through n = N(x), given that of n."""
        d = x - x.mean(1, keepdim=True) if kind == "layer" else x
        r = torch.rsqrt(d.square().mean(1, keepdim=True) + EPS)
        g = g - n * (g * n).mean(1, keepdim=True)
        if kind == "layer":
            g = g - g.mean(1, keepdim=True)
        return g * r
    gh = s["gh"].float()
    n = _norm32(s["x"], case["norm"])
    dx = s["gx"] + back(s["x"], n, gh * mul, case["norm"])
    du = gate * dx
    out = {"dx": dx, "dgate": _column_sums(dx * u, case)}
    if _post(case):
        out["dy"] = back(y, n_post, du * w, case["post"]).to(torch.bfloat16)
        out["dpost_w"] = (du * n_post).sum(0)
    else:
        out["dy"] = du.to(torch.bfloat16)
    if case["mod"]:
        out["dscale"], out["dshift"] = _column_sums(gh * n, case), _column_sums(gh, case)
    else:
        out["dw"] = (gh * n).sum(0)
        if case["norm"] == "layer":
            out["db"] = gh.sum(0)
    return out


# ---------------------------------------------------------------- one pass
def run(s):
    if not own:
        return _plain(s)
    from paper_2607_28144_amd import dit, mx
    case = s["case"]
    k = case["kind"]
    if k == "linear":
        return mx.linear_fwd(s["a"], s["w"], s["b"], epilogue="bias_gelu" if case["gelu"] else "bias")
    if k == "cache":
        if not case["append"]:
            return mx.attn_cache_fwd(s["q"], s["cache"], s["lens"])
        s["cache"].append(s["k_new"], s["v_new"], s["start"])
        return (*mx.attn_cache_fwd(s["q"], s["cache"], s["lens"]), *s["cache"].values(torch.bfloat16))
    vectors = {n: s[n] for n in ("gate", "scale", "shift", "w", "b", "post_w") if n in s}
    if k == "norm":
        return dit.residual_norm_fwd(s["x"], s["y"], norm=case["norm"], post=_post(case), group_rows=case["group"],
                                     eps=EPS, **vectors)
    vectors.pop("shift", None)
    g = dit.residual_norm_bwd(s["x"], s["y"], s["gh"], s["gx"], norm=case["norm"], post=_post(case),
                              group_rows=case["group"], eps=EPS, **vectors)
    names = ["dx", "dgate", "dy"] + (["dpost_w"] if _post(case) else [])
    names += ["dscale", "dshift"] if case["mod"] else ["dw", "db"] if case["norm"] == "layer" else ["dw"]
    return {n: getattr(g, n) for n in names}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    k = case["kind"]
    if k == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": 2 * M * K + N * K // 2 + N * K // 32 + 2 * N + 2 * M * N, "flops": 2 * M * N * K}
    if k == "cache":
        B, S, H, Hkv, D = (case[n] for n in ("B", "S", "H", "Hkv", "D"))
        n, token = sum(_lens(case)), Hkv * D // 2 + Hkv * D // 32
        new = 0
        if case["append"]:  # new tokens, and the cache's values as they are after the step
            new = B * S * (4 * Hkv * D + 2 * token) + B * case["cap"] * (2 * token + 4 * Hkv * D)
        return {"bytes": 4 * B * S * H * D + 4 * B * H * S + 2 * n * token + new, "flops": 4 * S * H * D * n}
    rows, C, G = case["rows"], case["C"], _groups(case)
    vectors = (3 if case["mod"] else 1) * 4 * G * C + 2 * C * ((not case["mod"]) * 2 + (_post(case) is not None))
    if k == "norm":
        return {"bytes": 12 * rows * C + vectors, "flops": 15 * rows * C}
    return {"bytes": 18 * rows * C + 2 * vectors, "flops": 30 * rows * C}


# ---------------------------------------------------------------- the same in 64 bits
def _mx64(x):
    """The values that x [..., n] has in MXFP4, from the definition: steps of 1/2 below 2, of 1 below 4, of 2 up to 6."""
    x = x.double()
    n = x.shape[-1]
    b = torch.cat([x, x.new_zeros(x.shape[:-1] + (-n % 32,))], -1).reshape(x.shape[:-1] + (-1, 32))
    top = b.abs().max(-1, keepdim=True).values
    scale = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.where(top > 0, top, 1.0)) + 1e-9) - 2, min=-127))
    m = (b / scale).abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0)).double()
    m = torch.clamp(torch.round(m / step) * step, max=6)
    return (torch.sign(b) * m * scale).reshape(x.shape[:-1] + (-1,))[..., :n]


def exact(case, seed):
    s = _inputs(case, seed)
    k = case["kind"]
    if k == "linear":
        y = torch.mm(_mx64(s["a"]), _mx64(s["w"]).t().contiguous()) + s["b"].double()
        return y * torch.sigmoid(math.sqrt(8 / math.pi) * (y + 0.044715 * y * y * y)) if case["gelu"] else y
    if k == "cache":
        B, S, H, Hkv, D, cap = (case[n] for n in ("B", "S", "H", "Hkv", "D", "cap"))
        keys, values = s["k"].clone(), s["v"].clone()
        if case["append"]:
            for b in range(B):
                for i in range(max(0, S - cap), S):
                    at = (int(s["start"][b]) + i) % cap
                    keys[b, at], values[b, at] = s["k_new"][b, i], s["v_new"][b, i]
        keys, values = _mx64(keys), _mx64(values)
        scale = float(torch.tensor(1.0 / math.sqrt(D), dtype=torch.float32))
        o = torch.empty((B, S, H, D), dtype=torch.float64, device=DEV)
        lse = torch.empty((B, H, S), dtype=torch.float64, device=DEV)
        for b in range(B):
            n = _lens(case)[b]
            for h in range(H):
                z = torch.mm(s["q"][b, :, h].double(), keys[b, :n, h // (H // Hkv)].t().contiguous()) * scale
                lse[b, h] = torch.logsumexp(z, 1)
                o[b, :, h] = torch.mm(torch.exp(z - lse[b, h][:, None]), values[b, :n, h // (H // Hkv)].contiguous())
        return (o, lse, keys, values) if case["append"] else (o, lse)
    d = {n: t.double() for n, t in s.items()}
    rows, C, G = case["rows"], case["C"], _groups(case)
    group = torch.arange(rows, device=DEV) // case["group"] if case["group"] else torch.zeros(rows, dtype=torch.long, device=DEV)

    def norm(x, kind):
        mean = x.sum(1) / C if kind == "layer" else torch.zeros(rows, dtype=torch.float64, device=DEV)
        z = x - mean[:, None]
        sigma = torch.sqrt((z * z).sum(1) / C + EPS)
        return z / sigma[:, None], sigma[:, None]

    def back(g, unit, sigma, kind):
        g = g - unit * ((g * unit).sum(1) / C)[:, None] - (g.sum(1, keepdim=True) / C if kind == "layer" else 0)
        return g / sigma

    def group_sums(t):
        return torch.zeros((G, C), dtype=torch.float64, device=DEV).index_add_(0, group, t)
    y_unit, y_sigma = norm(d["y"], case["post"]) if _post(case) else (d["y"], None)
    u = y_unit * d["post_w"] if _post(case) else d["y"]
    mul = 1 + d["scale"][group] if case["mod"] else d["w"]
    if k == "norm":
        x = d["x"] + d["gate"][group] * u
        h = norm(x, case["norm"])[0] * mul
        if case["mod"]:
            h = h + d["shift"][group]
        elif case["norm"] == "layer":
            h = h + d["b"]
        return x, h
    unit, sigma = norm(d["x"], case["norm"])
    dx = d["gx"] + back(d["gh"] * mul, unit, sigma, case["norm"])
    du = d["gate"][group] * dx
    out = {"dx": dx, "dgate": group_sums(dx * u)}
    if _post(case):
        out["dy"] = back(du * d["post_w"], y_unit, y_sigma, case["post"])
        out["dpost_w"] = (du * y_unit).sum(0)
    else:
        out["dy"] = du
    if case["mod"]:
        out["dscale"], out["dshift"] = group_sums(d["gh"] * unit), group_sums(d["gh"])
    else:
        out["dw"] = (d["gh"] * unit).sum(0)
        if case["norm"] == "layer":
            out["db"] = d["gh"].sum(0)
    return out
