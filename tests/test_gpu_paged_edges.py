"""Infinities and NaN in values of the paged cache that queries see."""
import copy

import numpy as np
import pytest

from paged_cases import Case
from test_gpu_paged import bf16, check, held, ints, paged

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


# rows, H, heads, D, page: tiles of 16, 32, 64 and 256 rows
SEEN = [(9, 4, 2, 128, 32), (30, 2, 2, 64, 16), (60, 6, 6, 128, 64), (300, 2, 2, 128, 32), (300, 4, 2, 64, 16)]


@pytest.mark.parametrize("rows,H,heads,D,page", SEEN)
@pytest.mark.parametrize("bits", [0x7fc0, 0x7f80])
@pytest.mark.parametrize("listed", [False, True])
def test_a_value_that_all_see_leaves_the_rest_of_the_row(rows, H, heads, D, page, bits, listed):
    """An infinity or NaN in one channel of an early value: the other channels come out to the last bit as without it."""
    n = rows + 700
    c = Case([rows, 1], [n, 90], H, heads, D, page, seed=rows)
    d = copy.copy(c)
    d.v = c.v.copy()
    d.v[c.table[0, 5 // page], :, 5 % page, 3] = bits
    if listed:
        lists = np.tile(np.arange(-(-n // page), dtype=np.int32), (c.T // 16 + 2, heads, 1))
        run = lambda x: paged().attn_pages_fwd(bf16(x.q), *held(x), ints(lists), 16, out_dtype=torch.float32)  # noqa: E731
    else:
        run = lambda x: paged().attn_fwd(bf16(x.q), *held(x), out_dtype=torch.float32)  # noqa: E731
    (co, cl), (o, lse) = run(c), run(d)
    bad = o[:rows, :, 3]
    assert bool((torch.isnan(bad) if bits == 0x7fc0 else torch.isposinf(bad)).all())
    o[:rows, :, 3] = co[:rows, :, 3]
    assert torch.equal(o, co) and torch.equal(lse, cl)


@pytest.mark.parametrize("rows,H,heads,D,page", SEEN)
@pytest.mark.parametrize("listed", [0, 1, 2])
def test_a_value_at_every_border_of_a_tile(rows, H, heads, D, page, listed):
    """A NaN in one value of the chunk, at the borders of its tiles and units: of no account to the rows before it, and to
    those from it on only in its channel.  listed: the pages from a list, in falling order, or each of them named twice."""
    n = rows + 700
    c = Case([rows], [n], H, heads, D, page, seed=rows + D)
    count = -(-n // page)
    lists = None
    if listed:
        lists = np.tile(np.repeat(np.arange(count, dtype=np.int32)[::-1], listed), (c.T // 128 + 1, heads, 1))
    cached = held(c)
    q, v = bf16(c.q), cached[0].v
    for i in sorted({0, 1, 15, 16, 17, rows // 2, min(rows, 255), min(rows, 256), rows - 1}):
        if i >= rows:
            continue
        place = n - rows + i
        at = (int(c.table[0, place // page]), slice(None), place % page, 7)
        keep = v[at].clone()
        v[at] = float("nan")
        if listed:
            o, lse = paged().attn_pages_fwd(q, *cached, ints(lists), 128, out_dtype=torch.float32)
        else:
            o, lse = paged().attn_fwd(q, *cached, out_dtype=torch.float32)
        v[at] = keep
        assert bool(torch.isnan(o[i:, :, 7]).all())
        if listed:
            co, _ = paged().attn_pages_fwd(q, *cached, ints(lists), 128, out_dtype=torch.float32)
        else:
            co, _ = paged().attn_fwd(q, *cached, out_dtype=torch.float32)
        o[i:, :, 7] = co[i:, :, 7]
        check(f"border {i} of {rows} listed={listed}", o, lse, c, True, selected=lists, q_block=128, f32=True)
