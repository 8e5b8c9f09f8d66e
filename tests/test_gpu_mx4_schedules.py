"""Whole schedules on registered 4-bit rows, epoch by epoch, and sets of other kinds registered in between."""
import numpy as np
import pytest

from tests import mx4_reference as R
from tests import parity as P
from tests.test_gpu_mx4 import dev, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("n,rows,cols,dim,cooling", [(700, 10, 12, 40, "linear"), (700, 10, 12, 40, "exponential"), (3000, 17, 13, 300, "linear"),
                                                     (9000, 30, 25, 64, "exponential"), (600, 9, 8, 1100, "linear")])
def test_every_epoch_of_a_schedule(oracle, n, rows, cols, dim, cooling):
    """Each snapshot is what one epoch at the schedule's radius makes of the snapshot before it: the same nodes, the same update."""
    rng = np.random.default_rng(n + dim)
    epochs, radius0 = 5, 0.4 * min(rows, cols)
    means = rng.standard_normal((8, dim))
    x = R.quantize(means[rng.integers(0, 8, n)] + 0.2 * rng.standard_normal((n, dim)))
    X = R.values(*x, dim)
    W = rng.standard_normal((rows * cols, dim)).astype(np.float32)
    som = make(rows, cols, dim, W)
    last, um, codebooks, all_bmus = som.train_snapshots(dev(x), epochs, radius0=radius0, radiusN=0.7, snapshots=2, cooling=cooling)
    assert torch.equal(all_bmus[-1], last) and torch.equal(codebooks[-1], som.codebook)
    before = W
    for e in range(epochs):
        b, after = all_bmus[e].cpu().numpy(), codebooks[e].cpu().numpy()
        assert np.array_equal(b, R.nearest(X, R.values(*R.quantize(before), dim))), e
        S, C = oracle.accumulate_dense(X.astype(np.float32), b, som.k)
        P.check_codebook(oracle, S, C, before, after, rows, cols, 0, 0, oracle.cool(radius0, 0.7, epochs, e, oracle.COOLING[cooling]))
        before = after
    assert torch.equal(um[-1].reshape(-1), som.umatrix().reshape(-1))
    som.codebook.copy_(P.to_dev(W))
    assert torch.equal(som.train(dev(x), epochs, radius0=radius0, radiusN=0.7, cooling=cooling), last)
    assert torch.equal(som.codebook, codebooks[-1])
    som.close()


def test_kinds_of_data_take_turns():
    """4-bit, dense and sparse sets registered one after the other on one map give what each gives on a map of its own."""
    rng = np.random.default_rng(41)
    rows, cols, dim = 11, 9, 48
    W = rng.standard_normal((rows * cols, dim)).astype(np.float32)
    sets = []
    for n in (400, 900):
        X = rng.standard_normal((n, dim)).astype(np.float32)
        X[rng.random((n, dim)) < 0.7] = 0.0
        at = np.nonzero(X)
        indptr = np.concatenate([[0], np.cumsum((X != 0).sum(1))]).astype(np.int64)
        sets += [dev(R.quantize(X)), P.to_dev(X), (P.to_dev(indptr), P.to_dev(at[1].astype(np.int32)), P.to_dev(X[at]))]
    sets = [sets[i] for i in (0, 1, 0, 2, 3, 5, 4, 3)]
    one = make(rows, cols, dim, W)
    for data in sets:
        own = make(rows, cols, dim, W)
        want_b = own.train(data, 3)
        one.codebook.copy_(P.to_dev(W))
        got_b = one.train(data, 3)
        assert torch.equal(got_b, want_b)
        if isinstance(data, tuple) and len(data) == 3:        # (sparse sums by atomics: their order is not fixed)
            assert torch.allclose(one.codebook, own.codebook, rtol=1e-5, atol=1e-6)
        else:
            assert torch.equal(one.codebook, own.codebook)
        own.close()
    one.close()
