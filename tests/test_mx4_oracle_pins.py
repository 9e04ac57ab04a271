"""oracle/mx4_oracle.py against hand-worked cases, the format's facts and a second way of rounding (no GPU)."""
import numpy as np
import pytest

from oracle import mx4_oracle as mo


def block(*first):
    x = np.zeros((1, 32))
    x[0, :len(first)] = first
    return x


def test_by_hand():
    # the largest is 5: floor(log2) = 2, scale 2^0; ties at 0.25, 0.75, 1.25, 1.75, 2.5, 3.5 and 5 go to the even code
    x = block(5.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.25, -0.75, 0.2500001, 4.999, 3.0)
    codes, scales = mo.quantise(x)
    assert scales[0, 0] == 127
    assert list(mo.values(codes, scales)[0, :12]) == [4, 0, 1, 1, 2, 2, 4, 0, -1, 0.5, 4, 3]
    # 7.9 lies above 6 and is cut off; a scale of 2^-3
    codes, scales = mo.quantise(block(7.9 / 8, -0.75 / 8))
    assert scales[0, 0] == 124 and list(mo.values(codes, scales)[0, :2]) == [0.75, -0.125]


def test_scales():
    for value, byte in ((0.0, 0), (4.0, 127), (7.99, 127), (8.0, 128), (1.0, 125), (2.0 ** -125, 0), (2.0 ** -124, 1), (2.0 ** -133, 0), (2.0 ** 127, 252), (np.inf, 255), (np.nan, 255)):
        assert mo.quantise(block(1e-300, value))[1][0, 0] == byte, value
    assert np.isnan(mo.values(*mo.quantise(block(1.0, np.nan)))).all()


def test_subnormal_blocks_keep_what_they_can():
    x = block(2.0 ** -126, 2.0 ** -133, -2.0 ** -128)
    assert list(mo.values(*mo.quantise(x))[0, :3]) == [2.0 ** -126, 0.0, -2.0 ** -128]   # steps of 2^-128


def test_rounding_a_second_way():
    r = np.random.default_rng(0)
    x = r.standard_normal((40, 96)) * np.exp2(r.integers(-20, 20, (40, 1)))
    got = mo.rounded(x)
    for row in range(40):
        for b in range(3):
            v = x[row, 32 * b:32 * b + 32]
            two = 2.0 ** (np.floor(np.log2(np.abs(v).max())) - 2)
            for k, a in enumerate(np.abs(v) / two):
                step = 0.5 if a < 2 else 1 if a < 4 else 2
                want = min(np.round(a / step) * step, 6.0) * two
                assert abs(got[row, 32 * b + k]) == want
    assert (np.sign(got) * np.sign(x) >= 0).all()


def test_layout():
    r = np.random.default_rng(1)
    x = r.standard_normal((70, 1040))
    codes, scales = mo.quantise(x)
    assert codes.shape == (70, 33, 32) and scales.shape == (70, 33)
    bytes_ = mo.pack(codes)
    assert bytes_.shape == (70, 528) and bytes_[3, 5] == codes[3, 0, 10] | codes[3, 0, 11] << 4
    s = mo.place_scales(scales, 1040)
    assert s.size == 3 * 128 * 16 and s[((17 // 16) * 128 + 69) * 16 + 4 * 1 + 0] == scales[69, 17] and s[(2 * 128 + 2) * 16 + 0] == scales[2, 32]
    assert (s.reshape(3, 128, 16)[:, 70:] == 127).all() and (s.reshape(3, 128, 16)[2, :, 1:] == 127).all()


def test_linear_on_exact_values():
    """Values that the format holds come through: a block's largest is 4 or 6."""
    r = np.random.default_rng(2)
    exact = lambda shape: mo.GRID[r.integers(0, 8, shape)] * r.choice([-1, 1], shape)
    X, W, dY = exact((64, 64)), exact((32, 64)), exact((64, 32))
    for a in (X, W, dY):     # every block of 32, either way, holds a 4
        a[::32, :], a[:, ::32] = 4, 4
    assert np.array_equal(mo.linear_fwd(X, W), X @ W.T)
    dX, dW = mo.linear_bwd(X, W, dY)
    assert np.array_equal(dX, dY @ W) and np.array_equal(dW, dY.T @ X)
