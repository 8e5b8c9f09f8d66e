"""Microscaled 4-bit rows in numbers that take more than one launch."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def make(dim):
    from paper_1305_1422_amd import Som
    return Som(1, 1, dim, seed=1)


def test_product_of_more_rows_than_a_launch_holds():
    """2^30 + 77 rows of a: 2^23 + 1 rows of tiles, and 2^32 threads are more than HIP takes.  The rows of b pick one element each, so that
    the products are the values of a, exact in bf16."""
    from paper_1305_1422_amd import Mx4
    n, picks = (1 << 30) + 77, (0, 17, 31)
    gen = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 256, (n, 16), dtype=torch.uint8, device="cuda", generator=gen)
    scales = torch.randint(120, 128, (n, 1), dtype=torch.uint8, device="cuda", generator=gen)
    b = torch.zeros((3, 16), dtype=torch.uint8, device="cuda")
    for j, c in enumerate(picks):
        b[j, c // 2] = 0x20 if c % 2 else 0x02                # 1.0
    som = make(32)
    out = som.products_mx4(Mx4(codes, scales), Mx4(b, torch.full((3, 1), 127, dtype=torch.uint8, device="cuda")), torch.bfloat16)
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float32, device="cuda")
    step = 1 << 26
    for lo in range(0, n, step):
        power = torch.exp2(scales[lo:lo + step, 0].float() - 127.0)
        for j, c in enumerate(picks):
            byte = codes[lo:lo + step, c // 2]
            want = level[(byte >> 4 if c % 2 else byte & 15).int()] * power
            assert torch.equal(out[lo:lo + step, j].float(), want), (lo, j)
    som.close()


def test_quantisation_of_more_blocks_than_a_launch_holds():
    """2^28 + 1,000 blocks: rows of one feature, whose values are 4 or 6 times their block's power of two."""
    n = (1 << 28) + 1000
    gen = torch.Generator(device="cuda").manual_seed(2)
    e = torch.randint(-30, 31, (n,), dtype=torch.int8, device="cuda", generator=gen)
    more = torch.randint(0, 4, (n,), dtype=torch.uint8, device="cuda", generator=gen)      # bit 0: 6 for 4; bit 1: negative
    x = (torch.exp2(e.float()) * (1.0 + 0.5 * (more & 1)) * (1.0 - (more & 2).float())).to(torch.bfloat16).reshape(n, 1)
    som = make(1)
    mx = som.quantize_mx4(x)
    assert torch.equal(mx.scales[:, 0], (e.int() - 2 + 127).to(torch.uint8))
    assert torch.equal(mx.codes[:, 0], 6 + (more & 1) + ((more & 2) << 2))
    assert not mx.codes[:, 1:].any()
    assert torch.equal(som.dequantize_mx4(mx, torch.bfloat16), x)
    som.close()
