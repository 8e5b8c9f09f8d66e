"""Updates of a map of 2^24 nodes, the most there may be."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("kind", ["dense", "csr", "mx4"])
@pytest.mark.parametrize("n", [700, 300_000])
def test_update(kind, n):
    """Every node hears its own instances only: those that have some get their mean, the others stay as they were."""
    from paper_1305_1422_amd import Som
    side, dim = 4096, 2
    k = side * side
    gen = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randint(-6, 7, (n, dim), generator=gen, device="cuda").float()
    x[x.abs() == 5] = 0.0                                     # (values that 4 bits hold)
    node = torch.randint(0, k, (n,), dtype=torch.int32, generator=gen, device="cuda")
    node[:200] = k - 1 - torch.arange(200, dtype=torch.int32, device="cuda") % 3      # several chunks each, at the end of the map
    som = Som(side, side, dim, seed=1)
    som.set_neighborhood("bubble")
    before = som.codebook.clone()
    data = x
    if kind == "csr":
        data = (torch.arange(0, 2 * n + 1, 2, device="cuda"), torch.arange(2, dtype=torch.int32, device="cuda").repeat(n), x.reshape(-1).contiguous())
    elif kind == "mx4":
        data = som.quantize_mx4(x)
        assert torch.equal(som.dequantize_mx4(data), x)
    som.update(data, node, 0.5)
    S = torch.zeros((k, dim), dtype=torch.float64, device="cuda").index_add_(0, node.long(), x.double())
    C = torch.bincount(node.long(), minlength=k)[:, None]
    want = torch.where(C > 0, (S / C.clamp(min=1)).float(), before)      # (S is whole, so the quotient's rounding is the only one)
    assert torch.equal(som.codebook, want)
    som.close()
