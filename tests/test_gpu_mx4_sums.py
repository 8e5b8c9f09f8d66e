"""Sums of microscaled 4-bit rows whose blocks' scales lie far apart: a small row between large ones that cancel."""
import numpy as np
import pytest

from tests import mx4_reference as R
from tests import parity as P
from tests.test_gpu_mx4 import dev, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def update_alone(x, bmus, rows, cols, dim, W):
    """The code book after an update in which every node hears its own instances only."""
    som = make(rows, cols, dim, W)
    som.set_neighborhood("bubble")
    som.update(dev(x), P.to_dev(bmus), 0.5)
    got = som.codebook.double().cpu().numpy()
    som.close()
    return got


# few instances are gathered (up to 262,144 features in all), more of them added up by chunks, where rows of up to 32, 64, .. 512 and more
# features share a wavefront
@pytest.mark.parametrize("nodes,dim", [(20, 40), (3000, 32), (1500, 64), (900, 130), (400, 300), (300, 500), (200, 700), (150, 1000), (60, 2100)])
@pytest.mark.parametrize("apart", [10, 30, 45])
@pytest.mark.parametrize("rows_of_a_node", [3, 32])
def test_small_rows_between_large_ones(nodes, dim, apart, rows_of_a_node):
    """Pairs of rows that cancel, 2^apart above the one or two that are left.  fp64 sums of 15 values of 12 x 2^45 times the least
    step at most are exact (2^52.5 < 2^53); then S and the quotient are rounded to fp32: two half steps."""
    rng = np.random.default_rng(dim + apart)
    b = R.blocks(dim)
    codes, scales = R.random_rows(rng, rows_of_a_node * nodes, dim, 100, 104)
    codes, scales = codes.reshape(nodes, rows_of_a_node, 16 * b), scales.reshape(nodes, rows_of_a_node, b)
    pairs = (rows_of_a_node - 1) // 2
    scales[:, :2 * pairs] = 100 + apart
    signs = np.zeros(32 * b, np.uint8)
    signs[:dim] = 8
    codes[:, pairs:2 * pairs] = codes[:, :pairs] ^ (signs[0::2] | signs[1::2] << 4)
    order = np.concatenate([np.arange(pairs), np.arange(2 * pairs, rows_of_a_node), np.arange(pairs, 2 * pairs)])
    x = codes[:, order].reshape(-1, 16 * b), scales[:, order].reshape(-1, b)
    rows = nodes // 10
    bmus = np.repeat(np.arange(nodes, dtype=np.int32), rows_of_a_node)
    left = R.values(codes[:, 2 * pairs:].reshape(-1, 16 * b), scales[:, 2 * pairs:].reshape(-1, b), dim).reshape(nodes, -1, dim).sum(1)
    want = left / rows_of_a_node
    got = update_alone(x, bmus, rows, 10, dim, np.full((nodes, dim), 7.0, np.float32))
    assert np.all(np.abs(got - want) <= 2.0 ** -23 * (1 + 2.0 ** -20) * np.abs(want))


@pytest.mark.parametrize("nodes,dim", [(20, 40), (400, 300), (150, 1000)])
def test_sums_that_pass_the_range_of_fp32_on_their_way(nodes, dim):
    b = R.blocks(dim)
    codes = np.zeros((nodes, 3, 16 * b), np.uint8)
    codes[:, :, 0] = [0x7, 0x7, 0xf]                                        # 6, 6, -6 in the first element
    scales = np.full((nodes, 3, b), 252, np.uint8)                           # 6 x 2^125 = 1.5 x 2^127
    x = codes.reshape(-1, 16 * b), scales.reshape(-1, b)
    bmus = np.repeat(np.arange(nodes, dtype=np.int32), 3)
    got = update_alone(x, bmus, nodes // 10, 10, dim, np.full((nodes, dim), 7.0, np.float32))
    want = np.zeros((nodes, dim))
    want[:, 0] = 2.0 * 2.0 ** 125
    assert np.all(np.abs(got - want) <= 2.0 ** -23 * (1 + 2.0 ** -20) * want)


def test_gathered_and_chunked_sums_agree():
    """The same instances, once alone (gathered) and once among others on other nodes (by chunks): the same node."""
    rng = np.random.default_rng(5)
    dim, n = 100, 60
    x = R.random_rows(rng, n, dim, 90, 130)
    more = R.random_rows(rng, 6000, dim, 90, 130)
    W = np.zeros((100, dim), np.float32)
    few = update_alone(x, np.zeros(n, np.int32), 10, 10, dim, W)
    both = tuple(np.concatenate([a, c]) for a, c in zip(x, more))
    many = update_alone(both, np.concatenate([np.zeros(n), 1 + np.arange(6000) % 99]).astype(np.int32), 10, 10, dim, W)
    # the two chunks' sums are rounded to fp32, then the sum and the quotient on both sides
    size = np.abs(R.values(*x, dim)).sum(0) / n
    assert np.all(np.abs(few[0] - many[0]) <= 3 * 2.0 ** -23 * size)
