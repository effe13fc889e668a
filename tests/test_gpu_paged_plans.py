"""Attention over the paged cache by plans that are taken for few calls only, each
asked for with all that the call has, causal or not, against the fp64 oracle."""
import ctypes

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


def plan(c, causal, q_block=1, count=0):
    from paper_2607_28144_amd import _lib
    p = _lib.PagedAttnPlan()
    s = _lib.PagedAttnShape(c.B, c.T, c.H, c.heads, c.D, c.page, q_block, count, c.T, c.table.shape[1] * c.page, int(causal))
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    assert _lib.load().regenvc_paged_attn_plan_query(ctypes.byref(s), n_cu, ctypes.byref(p)) == 0
    return p


# rows, places, H, heads, D, rows of no sequence before and behind
ONE = [(600, 2100, 4, 4, 64, 0, 0), (600, 2100, 4, 4, 128, 0, 0), (1000, 1024, 2, 2, 128, 0, 0), (500, 1900, 4, 2, 64, 3, 9),
       (700, 1500, 6, 3, 128, 0, 100)]


@pytest.mark.parametrize("rows,places,H,heads,D,lead,tail", ONE)
def test_one_short_causal_sequence_in_ranges(rows, places, H, heads, D, lead, tail):
    """More new tokens than a quarter of the places: two workgroups to a compute unit, with keys in ranges."""
    c = Case([rows], [places], H, heads, D, 64, seed=rows + D, lead=lead, tail=tail)
    p = plan(c, True)
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    assert p.split == 1 and p.tile_rows == 256 and p.workgroups == 2 * n_cu
    o, lse = paged().attn_fwd(bf16(c.q), *held(c), out_dtype=torch.float32)
    check(f"one causal {(rows, places, H, heads, D)}", o, lse, c, True, f32=True)


@pytest.mark.parametrize("B", [256, 257, 300])
def test_one_long_sequence_among_more_than_are_cut(B):
    """One of 4000 places among short ones, some without rows: cut for up to 256 sequences, whole beyond them."""
    rows = [0 if b % 7 == 3 else 1 + b % 3 for b in range(B)]
    lens = [4000 if b == B - 2 else 3 + (11 * b) % 200 for b in range(B)]
    c = Case(rows, lens, 2, 1, 64, 64, seed=B)
    for causal in (True, False):
        assert plan(c, causal).split == (B <= 256)
        o, lse = paged().attn_fwd(bf16(c.q), *held(c), causal=causal, out_dtype=torch.float32)
        check(f"{B} sequences", o, lse, c, causal, f32=True)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows,lens", [([300, 40], [5000, 900]), ([1] * 20, [700 * (b + 1) for b in range(20)])])
def test_ranges_with_the_plan_of_the_call(rows, lens, causal):
    """Keys of several sequences in ranges, of every place and of listed pages, planned as the call plans."""
    c = Case(rows, lens, 4, 2, 64, 64, seed=len(rows))
    assert plan(c, causal).split == 1
    o, lse = paged().attn_fwd(bf16(c.q), *held(c), causal=causal, out_dtype=torch.float32)
    check(f"ranges {len(rows)}", o, lse, c, causal, f32=True)
    count, q_block = 40, 16
    assert plan(c, causal, q_block, count).split == 1
    lists = np.argsort(np.random.default_rng(3).random((c.T // q_block + c.B, 2, c.table.shape[1])))[:, :, :count].astype(np.int32)
    o, lse = paged().attn_pages_fwd(bf16(c.q), *held(c), ints(lists), q_block, causal, out_dtype=torch.float32)
    check(f"listed ranges {len(rows)}", o, lse, c, causal, selected=lists, q_block=q_block, f32=True)
