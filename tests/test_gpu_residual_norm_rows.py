"""The seam's gradients where a workgroup goes through several rows of several
waves each: the waves' exchange buffers from row to row, the next row's loads,
sums kept over rows, segments and whole groups, and rows of more than eight
waves.  Oracle and bounds are those of test_gpu_residual_norm."""
import ctypes

import pytest

from test_gpu_residual_norm import case, dit, run

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()



def plan(rows, C, group):
    """Workgroups of a backward call, and the segments of its groups (0: each group is one), from what their sums take."""
    from paper_2607_28144_amd import _lib
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    out = []
    for sums in ((0, 1), (1, 0)):
        n = ctypes.c_int64()
        assert _lib.load().regenvc_residual_norm_bwd_workspace(rows, C, group, *sums, n_cu, ctypes.byref(n)) == 0
        out.append(n.value // (4 * C))
    return out


# rows, C, norm, post, modulated, rows of a group; rows that a workgroup goes through, at least
CASES = [(1600, 2048, "rms", "rms", False, 0, 3), (6200, 1536, "layer", None, True, 1560, 8),
         (6200, 1536, "layer", "layer", True, 1560, 8), (6200, 1536, "rms", "layer", False, 0, 8),
         (3000, 1032, "layer", "rms", True, 0, 5), (1900, 2560, "rms", None, False, 0, 7),
         (1900, 4096, "layer", "layer", True, 700, 7), (700, 6144, "layer", "rms", False, 0, 2),
         (900, 8192, "rms", "layer", True, 450, 3), (900, 4104, "layer", None, True, 0, 3)]


@pytest.mark.parametrize("rows,C,norm,post,mod,group,through", CASES)
@pytest.mark.parametrize("f32", [False, True])
def test_rows_of_a_workgroup(rows, C, norm, post, mod, group, through, f32):
    blocks, segments = plan(rows, C, group)
    assert rows / blocks >= through - 0.5 and segments > 0
    t, v, how = case(rows, C, norm, post, mod=mod, group=group, f32=f32)
    run(t, v, how, f32)


@pytest.mark.parametrize("rows,C,group", [(1100, 1536, 1), (2000, 1544, 2), (900, 2056, 1), (700, 8192, 1), (1700, 1024, 1)])
@pytest.mark.parametrize("post", [None, "layer"])
def test_groups_of_a_workgroup(rows, C, group, post):
    """More groups than workgroups: each is one segment, and a workgroup takes several."""
    blocks, segments = plan(rows, C, group)
    assert segments == 0 and -(-rows // group) > blocks
    t, v, how = case(rows, C, "layer", post, group=group)
    run(t, v, how, False)


@pytest.mark.parametrize("rows,C,group", [(1600, 2048, 0), (6200, 1536, 1560), (900, 8192, 450)])
def test_repeated_bit_for_bit(rows, C, group):
    t, v, how = case(rows, C, "layer", "layer", group=group)
    v.pop("shift")
    a, b = (dit().residual_norm_bwd(t["x"], t["y"], t["gh"], t["gx"], **v, **how) for _ in range(2))
    for p, q in zip(a, b):
        assert (p is None and q is None) or torch.equal(p, q)
