"""CPU oracle of the microscaled 4-bit linear: quantisation to blocks of 32 with a scale of a power of two, the layout of codes and
scales, and the products of a linear.  Test infrastructure only: plain numpy, written from the definitions in include/f8.h; values
are exact in fp64, products unrounded.  Pinned in tests/test_mx4_oracle_pins.py."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def blocks_of(x):
    """x [rows, n] in whole blocks [rows, ceil(n / 32), 32], padded with zeros"""
    rows, n = x.shape
    nb = (n + 31) // 32
    b = np.zeros((rows, nb * 32))
    b[:, :n] = x
    return b.reshape(rows, nb, 32)


def quantise(x):
    """(codes [rows, blocks, 32] of 0 .. 15, scale bytes [rows, blocks]) of x [rows, n] along n; fp64 of finite or other bf16 values"""
    b = blocks_of(np.asarray(x, dtype=np.float64))
    finite = np.isfinite(b).all(axis=2)
    a = np.where(finite, np.abs(np.where(np.isfinite(b), b, 0)).max(axis=2), 0.0)
    _, e = np.frexp(a)                       # a = m 2^e, m in [0.5, 1): floor(log2(a)) = e - 1
    e = np.where(a > 0, np.maximum(e - 1 - 2, -127), -127)
    v = np.abs(np.where(np.isfinite(b), b, 0)) * np.exp2(-e.astype(np.float64))[:, :, None]
    # nearest of the grid, ties to the even code
    d = np.abs(v[..., None] - GRID)
    lo = d.argmin(axis=-1)                   # the lower of two equally near ones
    tie = (lo < 7) & (d[np.arange(d.shape[0])[:, None, None], np.arange(d.shape[1])[None, :, None], np.arange(32), np.minimum(lo + 1, 7)] == np.take_along_axis(d, lo[..., None], -1)[..., 0])
    code = np.where(tie & (lo % 2 == 1), lo + 1, lo)
    code = np.where(np.signbit(b), code + 8, code)
    return code.astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def values(codes, scales):
    """[rows, blocks * 32] in fp64"""
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0) * s[:, :, None]
    return v.reshape(codes.shape[0], -1)


def pack(codes):
    """bytes [rows, 16 * blocks]: element 2 i in the low nibble"""
    c = codes.reshape(codes.shape[0], -1)
    return (c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8)


def place_scales(scales, n):
    """the bytes in their order, bytes of no block 127"""
    rows, nb = scales.shape
    R, groups = (rows + 63) // 64 * 64, (n + 511) // 512
    out = np.full(groups * R * 16, 127, dtype=np.uint8)
    for r in range(rows):
        for b in range(nb):
            out[((b // 16) * R + r) * 16 + 4 * (b % 4) + (b % 16) // 4] = scales[r, b]
    return out


def rounded(x):
    """x [rows, n] as its codes stand for it"""
    return values(*quantise(x))[:, :x.shape[1]]


def linear_fwd(X, W):
    return rounded(X) @ rounded(W).T


def linear_bwd(X, W, dY):
    """(dX, dW): blocks along the contraction of each product"""
    return rounded(dY) @ rounded(W.T).T, rounded(dY.T) @ rounded(X.T).T
