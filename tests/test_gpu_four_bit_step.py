"""A step of a block that streams video in four bits, as a program runs it:
seam, QKV projection in MXFP4, rotary embedding, append to the MXFP4 cache and
attention over it, output projection, seam, feed-forward in MXFP4 -- each stage
against the fp64 oracle of its own operation on the inputs that it got (so that
a code that flips at a rounding border in one stage is not an error of the
next), the whole captured into a graph and replayed, and the seams' gradients.
"""
import numpy as np
import pytest

import oracle
from oracle import dit as odit
from oracle import mx as omx
from oracle import residual_norm as orn
from paper_2607_28144_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

C, F, HEADS, D = 512, 1088, 4, 128
GRID = (3, 4, 10)           # frames, rows, columns; a step brings one frame
S = GRID[1] * GRID[2]
CAP = 2 * S                 # the cache keeps two frames


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def host(t):
    return t.double().cpu().numpy()


class Step:
    def __init__(self):
        from paper_2607_28144_amd import api, dit, mx
        self.api, self.dit, self.mx = api, dit, mx
        g = torch.Generator(device="cuda")
        g.manual_seed(3)

        def r(*shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
            return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)
        self.weights = {"qkv": r(3 * C, C, std=0.05), "o": r(C, C, std=0.05), "up": r(F, C, std=0.05), "down": r(C, F, std=0.05)}
        self.bias = {n: r(w.shape[0], std=0.05) for n, w in self.weights.items()}
        self.q = {n: mx.quantize(w) for n, w in self.weights.items()}
        self.wqn, self.wkn, self.post = r(C, std=0.1, mean=1.0), r(C, std=0.1, mean=1.0), r(C, std=0.1, mean=1.0)
        self.mod = r(6 * C, std=0.3, dtype=torch.float32)
        self.cache = mx.KvCache(1, CAP, HEADS, D)
        self.x = torch.empty(S, C, device="cuda")
        self.y = torch.empty(S, C, dtype=torch.bfloat16, device="cuda")
        self.start, self.lens = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
        self.r = r

    def part(self, i):
        return self.mod[i * C:(i + 1) * C]

    def run(self, frame, x=None):
        """One frame's tokens: self.x and the branch output self.y to the stream after the feed-forward."""
        t = {}
        t["x1"], t["h1"] = self.dit.residual_norm_fwd(self.x, self.y, post="rms", post_w=self.post, gate=self.part(2),
                                                      scale=self.part(1), shift=self.part(0))
        t["qkv"] = self.mx.linear_fwd(t["h1"], self.q["qkv"], self.bias["qkv"])
        v = t["qkv"].view(1, S, 3, HEADS, D)
        t["qr"], t["kr"] = self.api.qk_norm_rope(v[:, :, 0], v[:, :, 1], self.wqn, self.wkn, GRID, token0=frame * S)
        self.cache.append(t["kr"], v[:, :, 2], self.start)
        t["att"], t["lse"] = self.mx.attn_cache_fwd(t["qr"], self.cache, self.lens)
        t["o"] = self.mx.linear_fwd(t["att"].view(S, C), self.q["o"], self.bias["o"])
        t["x2"], t["h2"] = self.dit.residual_norm_fwd(t["x1"], t["o"], gate=self.part(5), scale=self.part(4),
                                                      shift=self.part(3))
        t["f"] = self.mx.linear_fwd(t["h2"], self.q["up"], self.bias["up"], epilogue="bias_gelu")
        t["x3"] = t["x2"].clone()
        self.mx.linear_fwd(t["f"], self.q["down"], self.bias["down"], epilogue="gated_residual", gate=self.part(2), out=t["x3"])
        return t


def near(name, got, ref, tol):
    err = np.abs(host(got) - ref)
    ratio = float((err / tol).max())
    print(f"[step] {name}: {ratio:.3f} of the bound", flush=True)
    assert ratio <= 1.0, name


BF = 2.0 ** -8


def check_linear(name, s, got, a, w, gelu=False):
    A, W, b = omx.values(host(a)), omx.values(host(s.weights[w])), host(s.bias[w])
    y = A @ W.T + b
    slack = (2 * -(-A.shape[1] // 256) + 16) * 2.0 ** -24 * (np.abs(A) @ np.abs(W).T + np.abs(b))
    ref = odit.gelu_tanh(y) if gelu else y
    near(name, got, ref, BF * np.abs(ref) + 1.13 * slack + 1e-6)


def check_seam(name, s, x, y, xo, h, i, **how):
    rx, _ = orn.forward(host(x), host(y), gate=host(s.part(i + 2)), **how)
    near(name + " x", xo, rx, 2.0 ** -18 * (np.abs(host(x)) + 8 * np.abs(host(s.part(i + 2))) * (np.abs(host(y)) + 8)))
    _, rh = orn.forward(host(xo), np.zeros((S, C)), scale=host(s.part(i + 1)), shift=host(s.part(i)))
    near(name + " h", h, rh, BF * np.abs(rh) + 2.0 ** -17 * (np.abs(rh) + 8))


def test_stages_and_graph():
    s = Step()
    for frame in range(3):
        s.x.copy_(s.r(S, C, std=2.0, dtype=torch.float32))
        s.y.copy_(s.r(S, C))
        s.start.fill_(frame * S)
        s.lens.fill_(min(CAP, (frame + 1) * S))
        t = s.run(frame)
        torch.cuda.synchronize()
        check_seam(f"frame {frame} seam 1", s, s.x, s.y, t["x1"], t["h1"], 0, post="rms", post_w=host(s.post))
        check_linear(f"frame {frame} qkv", s, t["qkv"], t["h1"], "qkv")
        k, v = s.cache.values()
        place = frame * S % CAP
        vals = t["qkv"].view(1, S, 3, HEADS, D)[:, :, 2]
        assert np.array_equal(host(v[:, place:place + S]), omx.values(host(vals)))
        assert np.array_equal(host(k[:, place:place + S]), omx.values(host(t["kr"])))
        n = int(s.lens)
        ro, rl, mag = omx.attn(host(t["qr"]), host(k), host(v), [n], synth.default_scale(D))
        near(f"frame {frame} attention", t["att"], ro, (BF + 2.0 ** -10) * (mag + np.abs(ro)) + BF * np.abs(ro))
        near(f"frame {frame} lse", t["lse"], rl, np.full(rl.shape, 2e-4))
        check_linear(f"frame {frame} o", s, t["o"], t["att"].view(S, C), "o")
        check_seam(f"frame {frame} seam 2", s, t["x1"], t["o"], t["x2"], t["h2"], 3)
        check_linear(f"frame {frame} up", s, t["f"], t["h2"], "up", gelu=True)
    # the last frame's step again, captured: replays between eager runs give its bits
    ref = {n: a.clone() for n, a in t.items()}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = s.run(2)
    for _ in range(3):
        for a in out.values():
            a.zero_()
        g.replay()
        eager = s.run(2)
        torch.cuda.synchronize()
        for n in ref:
            assert torch.equal(out[n], ref[n]) and torch.equal(eager[n], ref[n]), n


def test_two_streams_at_once():
    """Two programs with a cache and a stream each, enqueued in turn, as each alone."""
    a, b = Step(), Step()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (a, b):
        s.x.normal_()
        s.y.normal_()
        s.lens.fill_(S)
    alone = [{n: t.clone() for n, t in s.run(0).items()} for s in (a, b)]
    torch.cuda.synchronize()
    for _ in range(3):
        outs = []
        for s, st in ((a, sa), (b, sb)):
            with torch.cuda.stream(st):
                outs.append(s.run(0))
        torch.cuda.synchronize()
        for got, ref in zip(outs, alone):
            for n in ref:
                assert torch.equal(got[n], ref[n]), n


def test_gradients_of_the_seams():
    """The step's two seams backward, chained: the second's dx is the first's gx; against the oracle's chain."""
    s = Step()
    s.x.normal_()
    s.y.normal_()
    s.lens.fill_(S)
    t = s.run(0)
    gh1, gh2 = s.r(S, C), s.r(S, C)
    gx = s.r(S, C, dtype=torch.float32)
    g2 = s.dit.residual_norm_bwd(t["x2"], t["o"], gh2, gx, gate=s.part(5), scale=s.part(4))
    g1 = s.dit.residual_norm_bwd(t["x1"], s.y, gh1, g2.dx, post="rms", post_w=s.post, gate=s.part(2), scale=s.part(1))
    r2 = orn.backward(host(t["x2"]), host(t["o"]), host(gh2), host(gx), gate=host(s.part(5)), scale=host(s.part(4)))
    r1 = orn.backward(host(t["x1"]), host(s.y), host(gh1), r2["dx"], post="rms", post_w=host(s.post), gate=host(s.part(2)),
                      scale=host(s.part(1)))
    for got, ref in ((g2, r2), (g1, r1)):
        for n in got._fields:
            z = getattr(got, n)
            if z is not None:
                near(f"{n}", z, ref[n], (2.0 ** -15 + S * 2.0 ** -24) * ref[f"|{n}|"] + (BF * np.abs(ref[n]) if n == "dy" else 0)
                     + 1e-30)


def test_a_row_of_any_stride():
    """A single row's stride, which torch leaves to chance, is not looked at."""
    s = Step()
    a = s.r(C)
    odd = torch.as_strided(a, (1, C), (1, 1))
    assert torch.equal(s.mx.linear_fwd(odd, s.q["o"]), s.mx.linear_fwd(a.view(1, C), s.q["o"]))
    x = torch.as_strided(s.r(C, dtype=torch.float32), (1, C), (3, 1))
    for got, ref in zip(s.dit.residual_norm_fwd(x, odd), s.dit.residual_norm_fwd(x.clone(), a.view(1, C))):
        assert torch.equal(got, ref)


def test_cache_tensors_stay():
    s = Step()
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        with pytest.raises(AttributeError):
            setattr(s.cache, name, getattr(s.cache, name).clone())
