"""Products of microscaled 4-bit rows by every kind of tile: values, rows that lie apart, blocks that are not numbers."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
# up to 64 rows of a come straight from memory; 128 x 128 tiles where 256 x 256 ones are fewer than the card's 256 compute units; else 128 x 256 for up to
# 512 features and 256 x 256 beyond
SIZES = {"few": (37, 300, 130), "narrow": (203, 331, 130), "narrow_long": (300, 131, 1_030), "low": (4_099, 4_101, 100), "low_512": (4_097, 4_111, 512),
         "wide": (4_100, 4_103, 1_030), "wide_whole": (4_096, 4_352, 1_024), "wide_513": (4_098, 4_177, 513)}


def random_rows(gen, n, dim, low, high):
    from paper_1305_1422_amd import Mx4
    blocks = (dim + 31) // 32
    codes = torch.randint(0, 256, (n, blocks, 16), dtype=torch.uint8, device="cuda", generator=gen)
    last = dim - 32 * (blocks - 1)
    codes[:, -1, (last + 1) // 2:] = 0
    if last % 2:
        codes[:, -1, last // 2] &= 15
    return Mx4(codes.reshape(n, 16 * blocks), torch.randint(low, high + 1, (n, blocks), dtype=torch.uint8, device="cuda", generator=gen))


def values(mx, dim):
    """fp64, from the format's definition."""
    n, blocks = mx.scales.shape
    level = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
    code = mx.codes.reshape(n, blocks, 16)
    v = torch.empty((n, blocks, 32), dtype=torch.float64, device="cuda")
    for u, nibble in enumerate((code & 15, code >> 4)):
        v[:, :, u::2] = level[(nibble & 7).int()] * (1.0 - 2.0 * (nibble >> 3))
    v *= torch.exp2(mx.scales.double() - 127.0).unsqueeze(2)
    v[mx.scales == 255] = float("nan")
    return v.reshape(n, 32 * blocks)[:, :dim].contiguous()


def make(dim):
    from paper_1305_1422_amd import Som
    return Som(1, 1, dim, seed=1)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("size", list(SIZES))
def test_products(size, kind):
    """Exact sums of blocks added one after the other in fp32: half a step of at most the sum of the magnitudes for each, then one rounding to
    the type (and the reference's own, 2^-53 for every feature)."""
    n, m, dim = SIZES[size]
    gen = torch.Generator(device="cuda").manual_seed(n + dim)
    a, b = random_rows(gen, n, dim, 118, 130), random_rows(gen, m, dim, 118, 126)
    som = make(dim)
    got = som.products_mx4(a, b, TYPES[kind]).double()
    va, vb = values(a, dim), values(b, dim)
    want, size = va @ vb.T.contiguous(), va.abs() @ vb.abs().T.contiguous()
    tol = ((dim + 31) // 32 * 2.0 ** -24 * (1 + 2.0 ** -20) + dim * 2.0 ** -53) * size
    tol = tol + HALF_STEP[kind] * (want.abs() + tol) + (2.0 ** -25 if kind == "fp16" else 0.0)      # (half of fp16's least step)
    over = want.abs() > 65504 * (1 + 2.0 ** -11) if kind == "fp16" else torch.zeros_like(want, dtype=torch.bool)
    assert bool((((got - want).abs() <= tol) | over).all())
    som.close()


# rows aligned to 16, 4 and 2 bytes (fp32: 16 and 4), whole vectors and not, by stride and by base
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("size", ["few", "narrow", "low", "wide", "wide_whole"])
@pytest.mark.parametrize("more,offset", [(0, 0), (1, 0), (2, 0), (8, 8), (8, 2), (8, 1), (7, 3)])
def test_rows_that_lie_apart(size, kind, more, offset):
    """One scale a side: every sum is exact in fp32 and rounded once.  What lies between the rows is left as it is."""
    n, m, dim = SIZES[size]
    gen = torch.Generator(device="cuda").manual_seed(m)
    a, b = random_rows(gen, n, dim, 127, 127), random_rows(gen, m, dim, 126, 126)
    stride = (m + 7) // 8 * 8 + more if more != 1 else m + 1
    wide = torch.full((offset + n * stride + 64,), 7.0, dtype=TYPES[kind], device="cuda")
    out = torch.as_strided(wide, (n, m), (stride, 1), offset)
    som = make(dim)
    som.products_mx4(a, b, out=out)
    want = (values(a, dim) @ values(b, dim).T.contiguous()).float().to(TYPES[kind])
    assert torch.equal(out, want)
    keep = torch.ones_like(wide, dtype=torch.bool)
    torch.as_strided(keep, (n, m), (stride, 1), offset).fill_(False)
    assert bool((wide[keep] == 7.0).all())
    som.close()


@pytest.mark.parametrize("size", list(SIZES))
def test_blocks_that_are_not_numbers_and_blocks_of_zeros(size):
    """A block with scale 255 makes its row's products NaN whatever its codes, zeros among them (what a block with an infinity is stored as); zeros
    under the largest scale add nothing."""
    n, m, dim = SIZES[size]
    blocks = (dim + 31) // 32
    gen = torch.Generator(device="cuda").manual_seed(dim)
    a, b = random_rows(gen, n, dim, 127, 127), random_rows(gen, m, dim, 126, 126)
    for mx, rows in ((a, n), (b, m)):
        at = blocks - 1
        mx.scales[1, at], mx.scales[rows - 1, 0], mx.scales[3, at], mx.scales[5, :] = 255, 255, 254, 254
        mx.codes[1, 16 * at:], mx.codes[3, 16 * at:], mx.codes[5] = 0, 0, 0
    som = make(dim)
    got = som.products_mx4(a, b)
    want = values(a, dim) @ values(b, dim).T.contiguous()
    nan = torch.zeros((n, m), dtype=torch.bool, device="cuda")
    nan[1], nan[n - 1], nan[:, 1], nan[:, m - 1] = True, True, True, True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(torch.isnan(want), nan)
    assert torch.equal(got[~nan].double(), want[~nan])
    som.close()
