"""Mean keys of the paged cache that lie next to a tie of the rounding."""
import numpy as np
import pytest

from oracle import dit as odit
from test_gpu_paged import ints, paged

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("old", [0, 3])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 128, 1024])
def test_means_beside_a_tie(page, D, old):
    """Means a little above or below the middle of two bf16 numbers, by less than an f32 holds: rounded once, to the nearer
    one.  page times 1 + 2^-8 + 2^-30 is page + page 2^-8 + page 2^-30, exact in bf16 each; and so on."""
    one = [(1, 2.0 ** -8, 2.0 ** -30), (1, 2.0 ** -8, -2.0 ** -30), (1, 3 * 2.0 ** -8, 2.0 ** -30), (1, 3 * 2.0 ** -8, -2.0 ** -30),
           (2.0 ** -100, 2.0 ** -108, 2.0 ** -132), (1, 2.0 ** -8, 0.0)]
    k = np.zeros((page, 2, D), np.float64)
    for c, parts in enumerate(one):
        for i, x in enumerate(parts):
            k[5 * i, :, c], k[5 * i, :, c + 8] = page * x, -page * x
    bits = odit.round_bf16(k)
    assert np.array_equal(bits, k)
    cache = paged().PagedCache.zeros(1, page, 2, D, means=True)
    x = torch.from_numpy(k).float().bfloat16().cuda()
    if old:  # part of the page from an earlier call
        paged().append(cache, ints([[0]]), ints([0, old]), ints([old]), x[:old], x[:old])
    paged().append(cache, ints([[0]]), ints([0, page - old]), ints([page]), x[old:], x[old:])
    exact = np.zeros((2, D))
    for c, (a, b, e) in enumerate(one):
        # the nearer neighbour, 2^-7 times the leading part apart; a tie to the even one
        low = a if b < 2.0 ** -7 * a else a * (1 + 2.0 ** -7)
        up = e > 0 or (e == 0 and low != a)
        exact[:, c] = low + up * a * 2.0 ** -7
        exact[:, c + 8] = -exact[:, c]
    assert np.array_equal(cache.means[0].double().cpu().numpy(), exact)
