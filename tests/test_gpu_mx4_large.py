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


@pytest.mark.parametrize("n,dim", [(1 << 21, 16_384), (5_000_003, 1_100)])
def test_scratch_of_a_search_is_bounded(n, dim):
    """Rows for which a search of all at once would take 1.4 and 1.1 GB besides the nodes: it is made in parts, and finds the same nodes."""
    from paper_1305_1422_amd import Mx4, Som
    k, kinds, blocks = 3, 1000, (dim + 31) // 32
    gen = torch.Generator(device="cuda").manual_seed(dim)
    few = torch.randint(0, 256, (kinds, 16 * blocks), dtype=torch.uint8, device="cuda", generator=gen)
    if dim % 32:
        few[:, 16 * (blocks - 1) + dim % 32 // 2:] = 0        # (an even number of features: whole bytes)
    which = torch.randint(0, kinds, (n,), device="cuda", generator=gen)
    x = Mx4(torch.empty((n, 16 * blocks), dtype=torch.uint8, device="cuda"), torch.full((n, blocks), 127, dtype=torch.uint8, device="cuda"))
    torch.index_select(few, 0, which, out=x.codes)
    w = Mx4(few[:k].flip(1).contiguous() if dim % 32 == 0 else few[k:2 * k].clone(), torch.full((k, blocks), 126, dtype=torch.uint8, device="cuda"))
    som = Som(1, k, dim, seed=1)
    xv = som.dequantize_mx4(Mx4(few, x.scales[:kinds].contiguous())).double()
    wv = som.dequantize_mx4(w).double()
    score = xv @ wv.T - 0.5 * (wv * wv).sum(1)                # (exact: one scale a side)
    want = score.argmax(1).int()
    bmus = torch.empty(n, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    som.bmus(x, bmus, w)
    torch.cuda.synchronize()
    taken = before - torch.cuda.mem_get_info()[0]
    assert taken <= (1 << 30) + (64 << 20), taken             # (the nodes' part and rounding to pages: a few MB)
    assert torch.equal(bmus, want[which])
    som.close()
