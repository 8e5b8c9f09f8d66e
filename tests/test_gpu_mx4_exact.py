"""Searches of 4-bit rows over the whole range of scales for which their decision is promised to be exact."""
import numpy as np
import pytest

from tests import mx4_reference as R
from tests.test_gpu_mx4 import dev, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def whole(codes, scales, dim, low):
    """The values in halves of 2^(low - 127), int64."""
    v = R.values(codes, np.full_like(scales, 127), dim) * 2.0
    return v.astype(np.int64) << (np.repeat(scales.astype(np.int64), 32, 1)[:, :dim] - low)


# a row of B blocks: products of scales within 2^39 / B, scales of a side within half as many powers of two
@pytest.mark.parametrize("dim,span", [(64, 19), (96, 18), (250, 18), (1000, 17), (2000, 16), (4096, 16)])
@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("kinds", [4, 150])
def test_search_is_exact_over_its_range(kinds, few, dim, span):
    """Nodes of a kind differ in their last block alone, which has the smallest scale; instances are like them: the nearest node is told by
    the last bits of the sums.  Compared in whole numbers, which stay below 2^62."""
    n, k = (3, 90) if few else (4000, 2500) if dim <= 250 else (1500, 600)      # (few: every score in fp64; else matrix cores first)
    rng = np.random.default_rng(dim + n + kinds)
    low, b = 110, R.blocks(dim)
    assert b * 2 ** (2 * span) <= 2 ** 39
    base = R.random_rows(rng, kinds, dim)
    base[1][:] = rng.choice([low, low + span // 2, low + span], base[1].shape)
    base[1][:, 0], base[1][:, -1] = low + span, low
    size = 16 * (b - 1)                                        # bytes before the last block

    def like(m):
        which = rng.integers(0, kinds, m)
        codes, scales = base[0][which].copy(), base[1][which].copy()
        last = R.random_rows(rng, m, dim - 32 * (b - 1), low, low)[0]
        keep = rng.random(last.shape) < 0.9
        codes[:, size:] = np.where(keep, codes[:, size:], last)
        return codes, scales

    x, w = like(n), like(k)
    som = make(1, k, dim)
    got = som.bmus(dev(x), nodes=dev(w)).cpu().numpy()
    som.close()
    xi, wi = (torch.from_numpy(whole(*t, dim, low)).cuda() for t in (x, w))
    half = (wi * wi).sum(1)
    want = np.empty(n, np.int32)
    for i in range(0, n, 50):
        score = 2 * (xi[i:i + 50, None] * wi[None]).sum(2) - half
        best = score.max(1, keepdim=True).values
        want[i:i + 50] = (score == best).int().argmax(1).cpu().numpy()
    assert np.array_equal(got, want)
