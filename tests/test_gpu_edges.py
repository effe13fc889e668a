"""Calls at the edge of what the MXFP4 cache and the seam take, through the torch
binding: a cache of no places, groups of more rows than there are (beyond 32 bits
too), and calls in place with another buffer at the same address."""
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("S", [1, 40, 300])
@pytest.mark.parametrize("D", [64, 128])
def test_a_cache_of_no_places(S, D):
    """Nothing to attend to, whatever the lengths say; nothing is kept of what is appended."""
    from paper_2607_28144_amd import mx
    c = mx.KvCache(2, 0, 3, D)
    q = torch.randn(2, S, 6, D, device="cuda").bfloat16()
    c.append(q[:, :, :3].contiguous(), q[:, :, 3:].contiguous())
    for lens in (None, torch.tensor([0, 5], dtype=torch.int32, device="cuda")):
        o, lse = mx.attn_cache_fwd(q, c, lens)
        assert bool((o == 0).all()) and bool(torch.isneginf(lse).all())
    assert c.values()[0].shape == (2, 0, 3, D)


@pytest.mark.parametrize("group_rows", [50, 51, (1 << 31) - 1, 1 << 31, (1 << 32) + 1, sys.maxsize])
def test_a_group_of_all_rows_or_more(group_rows):
    """... is one set of vectors for all rows, as group_rows=0 is."""
    from paper_2607_28144_amd import dit
    rows, C = 50, 1536
    x, gx = (torch.randn(rows, C, device="cuda") for _ in range(2))
    y, gh = (torch.randn(rows, C, device="cuda").bfloat16() for _ in range(2))
    gate, scale, shift = (torch.randn(C, device="cuda") for _ in range(3))
    a, b = (dit.residual_norm_fwd(x, y, gate=gate, scale=scale, shift=shift, group_rows=n) for n in (0, group_rows))
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    a, b = (dit.residual_norm_bwd(x, y, gh, gx, gate=gate, scale=scale, group_rows=n) for n in (0, group_rows))
    assert all(p is q is None or torch.equal(p, q) for p, q in zip(a, b))


def test_in_place_and_nothing_else_there():
    from paper_2607_28144_amd import dit
    from paper_2607_28144_amd._lib import RegenvcError
    x, y, gh, gx = (torch.randn(20, 512, device="cuda") for _ in range(4))
    keep = [t.clone() for t in (x, y, gh, gx)]
    for call in (lambda: dit.residual_norm_fwd(x, y, out=x, h=x), lambda: dit.residual_norm_fwd(x, x, out=x),
                 lambda: dit.residual_norm_bwd(x, y, gh, gx, dx=gx, dy=gx),
                 lambda: dit.residual_norm_bwd(x, y, gx, gx, dx=gx), lambda: dit.residual_norm_bwd(gx, y, gh, gx, dx=gx)):
        with pytest.raises(RegenvcError, match="overlaps"):
            call()
    assert all(torch.equal(a, b) for a, b in zip(keep, (x, y, gh, gx)))
