"""Microscaled 4-bit rows in numpy, fp64, from the format's definition (helpers of the tests)."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def blocks(dim):
    return (dim + 31) // 32


def quantize(x):
    """(codes, scales) of the float matrix x: floor(log2 of a block's largest magnitude) - 2, nearest level, ties to even codes."""
    n, dim = x.shape
    b = blocks(dim)
    p = np.zeros((n, 32 * b))
    p[:, :dim] = x
    sign = np.zeros((n, 32 * b), dtype=np.uint8)
    sign[:, :dim] = np.signbit(x)
    p, sign = p.reshape(n, b, 32), sign.reshape(n, b, 32)
    bad = ~np.isfinite(p).all(2)
    with np.errstate(invalid="ignore"):
        top = np.where(bad, 0.0, np.abs(p).max(2))
    e = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -127)
    s = np.clip(e, -127, 127) + 127
    t = np.abs(np.where(bad[:, :, None], 0.0, p)) * np.exp2(127.0 - s)[:, :, None]
    off = np.abs(t[..., None] - LEVELS)
    near = off == off.min(-1, keepdims=True)
    code = near.argmax(-1)                                   # the lower of two equally near levels ...
    odd_tie = (near.sum(-1) == 2) & (code % 2 == 1)          # ... unless its code is odd
    code = (code + odd_tie).astype(np.uint8) | (sign << 3)
    code[bad] = 0
    s = np.where(bad, 255, s).astype(np.uint8)
    return (code[:, :, 0::2] | (code[:, :, 1::2] << 4)).reshape(n, 16 * b).astype(np.uint8), s


def values(codes, scales, dim):
    n, b = scales.shape
    c = codes.reshape(n, b, 16)
    nib = np.empty((n, b, 32), dtype=np.int64)
    nib[:, :, 0::2], nib[:, :, 1::2] = c & 15, c >> 4
    v = LEVELS[nib & 7] * np.where(nib & 8, -1.0, 1.0) * np.exp2(scales.astype(np.float64) - 127.0)[:, :, None]
    v[scales == 255] = np.nan
    return v.reshape(n, 32 * b)[:, :dim]


def random_rows(rng, n, dim, low=118, high=130, zero_tail=True):
    """Random codes and scales (bytes low..high)."""
    b = blocks(dim)
    codes = rng.integers(0, 256, (n, b, 16), dtype=np.int64).astype(np.uint8)
    if zero_tail and dim % 32:
        last = dim - 32 * (b - 1)
        nib = np.empty((n, 32), dtype=np.uint8)
        nib[:, 0::2], nib[:, 1::2] = codes[:, -1] & 15, codes[:, -1] >> 4
        nib[:, last:] = 0
        codes[:, -1] = nib[:, 0::2] | (nib[:, 1::2] << 4)
    return codes.reshape(n, 16 * b), rng.integers(low, high + 1, (n, b)).astype(np.uint8)


def nearest(x, w):
    """Lowest index of the largest x.w - |w|^2 / 2 (exact in fp64 for values of this kind close enough in scale); a NaN node
    is never chosen, a NaN instance has node 0."""
    with np.errstate(invalid="ignore"):
        s = x @ w.T - 0.5 * (w * w).sum(1)
    s[np.isnan(s)] = -np.inf
    out = s.argmax(1).astype(np.int32)
    out[np.isnan(x).any(1)] = 0
    return out
