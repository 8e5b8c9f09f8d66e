"""Recorded calls on 4-bit rows that share a map's scratch with one another and with eager calls of other sizes."""
import numpy as np
import pytest

from tests import mx4_reference as R
from tests import parity as P
from tests.test_gpu_mx4 import dev, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dim,sizes", [(96, (3000, 9000, 20)), (1100, (700, 2500, 3))])
def test_graphs_recorded_before_and_after_scratch_has_grown(dim, sizes):
    """One graph's scratch is replaced before the next is recorded; they are replayed in turns, eager calls between them."""
    rng = np.random.default_rng(dim)
    rows, cols = 20, 25
    k = rows * cols
    w = R.quantize(rng.standard_normal((k, dim)))
    w[0][k // 2:], w[1][k // 2:] = w[0][:k - k // 2], w[1][:k - k // 2]        # copies far apart: the second pass has work
    xs = [R.quantize(rng.standard_normal((n, dim))) for n in sizes]
    want = [R.nearest(R.values(*x, dim), R.values(*w, dim)) for x in xs]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        som = make(rows, cols, dim)
        wd, xd = dev(w), [dev(x) for x in xs]
        bmus = [torch.empty(n, dtype=torch.int32, device="cuda") for n in sizes]
        outs = [torch.empty((n, k), dtype=torch.bfloat16, device="cuda") for n in sizes]
        graphs, products = [], []
        for i in range(len(sizes)):
            som.bmus(xd[i], bmus[i], wd)
            som.products_mx4(xd[i], wd, out=outs[i])
            products.append(outs[i].clone())
            stream.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                som.bmus(xd[i], bmus[i], wd)
                som.products_mx4(xd[i], wd, out=outs[i])
            graphs.append(g)
        big = dev(R.quantize(rng.standard_normal((3 * max(sizes), dim))))
        for step in range(4):
            for i in (0, 1, 2, 1, 0):
                bmus[i].fill_(-1)
                outs[i].zero_()
                graphs[i].replay()
                assert np.array_equal(bmus[i].cpu().numpy(), want[i]), (step, i)
                assert torch.equal(outs[i], products[i]), (step, i)
                if step == 1:
                    som.bmus(big, nodes=wd)
                elif step == 2:
                    som.products_mx4(big, wd)
                stream.synchronize()
        som.close()


@pytest.mark.parametrize("n,dim", [(400, 40), (5000, 200)])
def test_recorded_schedule_goes_on_from_where_it_stands(oracle, n, dim):
    """A recorded epoch replayed is one epoch after the other: each replay takes the code book that the one before it left."""
    rng = np.random.default_rng(n)
    rows, cols, radius = 14, 11, 2.0
    means = rng.standard_normal((7, dim))
    x = R.quantize(means[rng.integers(0, 7, n)] + 0.3 * rng.standard_normal((n, dim)))
    X, W = R.values(*x, dim), rng.standard_normal((rows * cols, dim)).astype(np.float32)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        som = make(rows, cols, dim, W)
        xd, b = dev(x), torch.empty(n, dtype=torch.int32, device="cuda")
        other = dev(R.quantize(rng.standard_normal((4 * n, dim))))
        som.train_epoch(xd, radius, bmus=b)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            som.train_epoch(xd, radius, bmus=b)
        som.codebook.copy_(P.to_dev(W))
        before = W
        for step in range(4):
            graph.replay()
            after, nodes = som.codebook.cpu().numpy().copy(), b.cpu().numpy().copy()
            assert np.array_equal(nodes, R.nearest(X, R.values(*R.quantize(before), dim))), step
            S, C = oracle.accumulate_dense(X.astype(np.float32), nodes, som.k)
            P.check_codebook(oracle, S, C, before, after, rows, cols, 0, 0, radius)
            som.bmus(other)                      # (a search may be of any size: its scratch is another)
            before = after
        stream.synchronize()
        som.close()
