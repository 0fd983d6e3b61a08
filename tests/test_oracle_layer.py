"""The oracle of the 4-bit form, the rotation and the adapters against hand-made values."""

import numpy as np
import pytest

from oracle import layer


def test_codes_of_a_block():
    x = np.zeros(32)
    x[:8] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -5.0]       # ties, all to the even code
    codes, scale = layer.quantise(x)
    assert scale.tolist() == [127]                               # largest in [4, 8): unscaled
    assert codes[:8].tolist() == [6, 0, 2, 2, 4, 4, 6, 8 + 6]
    assert layer.values(codes, scale)[:8].tolist() == [4, 0, 1, 1, 2, 2, 4, -4]


@pytest.mark.parametrize("largest, byte", [(6.0, 127), (7.0, 127), (7.01, 128), (8.0, 128), (3.9, 127), (3.4, 126),
                                           (0.0, 1), (1e-40, 1), (3e38, 252)])
def test_scale_of_a_block(largest, byte):
    x = np.zeros(32)
    x[5] = -largest
    assert layer.quantise(x)[1].tolist() == [byte]


def test_a_value_is_off_by_at_most_the_scale():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 64)) * 10.0 ** rng.uniform(-3, 3, (200, 1))
    codes, scale = layer.quantise(x)
    off = np.abs(layer.values(codes, scale) - x).reshape(200, 2, 32)
    assert np.all(off <= 2.0 ** (scale.astype(float) - 127)[..., None])
    most = np.abs(x).reshape(200, 2, 32).max(-1)
    assert np.all(off.max(-1) <= most / 3.5)


def test_rounding_outside_the_scales():
    # Above 7 x 2^125 the scale stays at 2^125 and values saturate, less than 2^126 off; below
    # 3.5 x 2^-126 it stays at 2^-126 and a value is off by at most 2^-127, up to 2^-128 all of it.
    for top, bound in ((7.0, 2.0 ** 125), (7.01, 2.0 ** 126), (7.999, 2.0 ** 126)):
        x = np.linspace(-top, top, 32)[None] * 2.0 ** 125
        codes, scale = layer.quantise(x)
        y = layer.values(codes, scale)
        assert scale[0, 0] == 252 and np.abs(y).max() == 6 * 2.0 ** 125
        assert np.abs(y - x).max() <= bound and np.abs(y - x).max() <= np.abs(x).max() / 3.5
    for top in (3.49, 2.0, 0.3, 0.25, 0.1, 2.0 ** -23):
        x = np.linspace(-top, top, 32)[None] * 2.0 ** -126
        codes, scale = layer.quantise(x)
        y = layer.values(codes, scale)
        assert scale[0, 0] == 1 and np.abs(y - x).max() <= 2.0 ** -127
        assert np.array_equal(y == 0, np.abs(x) <= 2.0 ** -128)


def test_an_odd_value_makes_its_block_nan():
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones((1, 2, 1, 64))
        x[0, 1, 0, 40] = bad
        y = layer.unpack(layer.pack(x), 1, 64)
        assert np.all(y[0, 0] == 1) and np.all(y[0, 1, 0, :32] == 1) and np.all(np.isnan(y[0, 1, 0, 32:]))


def test_rows_in_bytes():
    assert layer.row_bytes(8, 128) == 1088 and layer.row_bytes(1, 32) == 48 and layer.row_bytes(1, 64) == 80
    x = np.random.default_rng(2).standard_normal((3, 2, 2, 96))
    rows = layer.pack(x)
    assert rows.shape == (3, 208)
    y = layer.unpack(rows, 2, 96)
    assert np.array_equal(layer.pack(y), rows)                    # what it holds, it holds exactly


def test_rotation():
    x = np.zeros((1, 1, 6))
    x[0, 0] = [1, 2, 3, 4, 5, 6]
    t = np.pi / 2
    assert np.allclose(layer.rotate(x, [1], [t, 2 * t])[0, 0], [-3, -2, 1, -4, 5, 6])
    assert np.allclose(layer.rotate(x, [1], [t, 2 * t], True)[0, 0], [-2, 1, -3, -4, 5, 6])
    assert np.array_equal(layer.positions([2, 0, 1], [1, 0, 2], [4, 10, 7]), [8, 9, 6])


def test_adapters():
    x, w = np.eye(3), np.zeros((2, 3))
    a = np.array([[[1.0, 2, 3]], [[1.0, 1, 1]]])
    b = np.array([[[1.0], [10]], [[1.0], [-1]]])
    out = layer.adapter_linear(x, w, a, b, [1, 2], [1, -1], scales=np.array([1.0, 4]))[0]
    assert np.array_equal(out, [[4, -4], [0, 0], [0, 0]])
    out = layer.adapter_linear(x, w, a, b, [1, 2], [7, 0], bias=np.array([0.0, -25]), relu=True)[0]
    assert np.array_equal(out, [[0, 0], [2, 0], [3, 5]])
