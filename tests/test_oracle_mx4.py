"""Pins of the oracle's microscaled 4-bit matrices: hand-worked blocks, brute force over
the steps, invariants."""
import numpy as np
import pytest

from oracle import mx4


def _block(values):
    x = np.zeros((1, 32))
    x[0, :len(values)] = values
    return x


def test_hand_worked_block():
    # the largest magnitude 5 has exponent 2: b = 127, steps as they are
    v = [5.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.3, -4.9, 0.2, 2.4]
    codes, scale = mx4.quantize(_block(v))
    assert scale.shape == (1, 1, 8) and scale[0, 0].tolist() == [127, 0, 0, 0, 0, 0, 0, 0]
    got = mx4.dequantize(codes, scale)[0, :len(v)]
    # ties: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    assert got.tolist() == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, -0.5, -4.0, 0.0, 2.0]
    # low half first
    assert codes[0, 0] == 6 | 0 << 4 and codes[0, 1] == 2 | 2 << 4


def test_exponents():
    assert mx4.exponent_of([0.0, 1.0, 7.99, 8.0, 0.99, np.inf, np.nan]).tolist() == \
        [0, 125, 127, 128, 124, 255, 255]
    assert mx4.exponent_of([2.0 ** -126, 2.0 ** -149, 2.0 ** -124, 2.0 ** 127.99]).tolist() == \
        [0, 0, 1, 252]


@pytest.mark.parametrize("seed", range(4))
def test_nearest_by_brute_force(seed):
    g = np.random.default_rng(seed)
    x = g.normal(size=(7, 64)) * 2.0 ** g.integers(-130, 120, size=(7, 1))
    codes, scale = mx4.quantize(x)
    v = mx4.dequantize(codes, scale)
    for r in range(7):
        for blk in range(2):
            s = slice(32 * blk, 32 * blk + 32)
            unit = 2.0 ** (int(scale[0, r, blk]) - 127)
            grid = np.concatenate([mx4.STEPS, -mx4.STEPS]) * unit
            assert np.array_equal(np.abs(v[r, s] - x[r, s]),
                                  np.abs(x[r, s][:, None] - grid).min(1))
            top = np.abs(x[r, s]).max() / unit
            assert top < 8 and (top >= 4 or scale[0, r, blk] == 0)


def test_values_survive_a_second_rounding():
    g = np.random.default_rng(9)
    v = mx4.dequantize(*mx4.quantize(g.normal(size=(2, 5, 288))))
    codes, scale = mx4.quantize(v)
    assert np.array_equal(mx4.dequantize(codes, scale), v)
    assert codes.shape == (2, 5, 144) and scale.shape == (2, 2, 5, 8)
    assert (scale[:, 1, :, 1:] == 0).all()


def test_not_finite_blocks():
    x = np.ones((1, 96))
    x[0, 40], x[0, 95] = np.inf, np.nan
    codes, scale = mx4.quantize(x)
    assert scale[0, 0, :3].tolist() == [125, 255, 255] and (codes[0, 16:] == 0).all()
    v = mx4.dequantize(codes, scale)
    assert (v[0, :32] == 1).all() and np.isnan(v[0, 32:]).all()


def test_product_by_loops():
    g = np.random.default_rng(3)
    x, w = g.normal(size=(5, 32)), g.normal(size=(2, 4, 32))
    out, mag = mx4.grouped_product(x, w, [0, 2, 2, 4], [1, -1, 0])
    for r in range(4):
        for n in range(4):
            t = [x[r, i] * w[1 if r < 2 else 0, n, i] for i in range(32)]
            assert abs(out[r, n] - sum(t)) < 1e-12 and abs(mag[r, n] - sum(map(abs, t))) < 1e-12
    assert np.isnan(out[4]).all()
