"""Pins of the microscaled oracle: the formats' numbers, rounding and scales, and the
operators at values that are known."""
import numpy as np
import pytest

from oracle import mx


def test_e2m1_numbers_follow_from_the_format():
    for c in range(8):
        e, m = c >> 1, c & 1
        assert mx.NUMBERS["e2m1"][c] == (m * 0.5 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1))


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_nearest_code_on_every_number_midpoint_and_side(fmt):
    n = mx.NUMBERS[fmt]
    codes = np.arange(len(n))
    mid = (n[1:] + n[:-1]) / 2
    np.testing.assert_array_equal(mx.nearest_code(n, fmt), codes)
    np.testing.assert_array_equal(mx.nearest_code(mid, fmt), codes[:-1] + codes[:-1] % 2)
    np.testing.assert_array_equal(mx.nearest_code(mid * (1 + 1e-12), fmt), codes[1:])
    np.testing.assert_array_equal(mx.nearest_code(mid * (1 - 1e-12), fmt), codes[:-1])
    np.testing.assert_array_equal(mx.nearest_code(-n, fmt), codes + (128 if fmt == "e4m3" else 8))


@pytest.mark.parametrize("fmt,top,e", [("e4m3", 448.0, 0), ("e4m3", 449.0, 1), ("e4m3", 0.0, -117), ("e2m1", 6.0, 0),
                                       ("e2m1", np.nextafter(6.0, 7), 1), ("e2m1", 3.0, -1), ("e2m1", 1.0, -2), ("e2m1", 0.75, -3),
                                       ("e2m1", 0.0, -117), ("e2m1", 2.0 ** -140, -117), ("e2m1", 1.9 * 2.0 ** 127, 126)])
def test_scale_exponents(fmt, top, e):
    assert mx.exponent(np.array([top]), fmt)[0] == e
    if top > 6 * 2.0 ** -117:  # the smallest that holds it
        assert mx.NUMBERS[fmt][-1] * 2.0 ** e >= top > mx.NUMBERS[fmt][-1] * 2.0 ** (e - 1)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_quantise_and_back(fmt):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 96)) * 2.0 ** rng.integers(-30, 30, (5, 1))
    x[2, 40] = np.inf
    codes, scales = mx.quantise(x, fmt)
    y = mx.numbers(codes, scales, fmt)
    assert np.isnan(y[2, 32:64]).all() and scales[2, 1] == 255
    y[2, 32:64] = x[2, 32:64] = 0.0
    again, s2 = mx.quantise(np.where(np.isnan(y), 0, y), fmt)
    np.testing.assert_array_equal(mx.numbers(again, s2, fmt), y)       # numbers of the format stay
    top = np.abs(x.reshape(5, 3, 32)).max(-1, keepdims=True)
    # half of the largest step: 2^-4 (e4m3) or 2^-2 (e2m1) of a number's leading power, at most of the block's largest
    assert (np.abs(y - x).reshape(5, 3, 32) <= top * (2.0 ** -4 if fmt == "e4m3" else 2.0 ** -2)).all()
    np.testing.assert_array_equal(mx.unpack_e2m1(mx.pack_e2m1(codes % 16)), codes % 16)


def test_turning_adds_up_and_keeps_lengths():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 64))
    f, ax = [10000.0 ** (-2 * j / 32) for j in range(16)], [j % 3 for j in range(16)]
    p, q = rng.integers(0, 1000, (2, 3, 3))
    for adjacent in (False, True):
        both = mx.turned(mx.turned(x, p, ax, f, adjacent), q, ax, f, adjacent)
        np.testing.assert_allclose(both, mx.turned(x, p + q, ax, f, adjacent), atol=1e-12)
        np.testing.assert_allclose((both ** 2).sum(-1), (x ** 2).sum(-1))
        np.testing.assert_array_equal(both[..., 32:], x[..., 32:])
    one = mx.turned(np.eye(64)[None, :1].repeat(1, 0), np.array([[1]]), [0] * 32, [np.pi / 2] * 32, False)
    np.testing.assert_allclose(one[0, 0, [0, 32]], [0, 1], atol=1e-15)


def test_norm_and_gate_at_known_values():
    np.testing.assert_allclose(mx.norm(np.array([[3.0, 4.0]]), np.array([1.0, 2.0]), 0.0), [[3 / np.sqrt(12.5), 8 / np.sqrt(12.5)]])
    np.testing.assert_allclose(mx.gated(np.array([2.0, 1.0]), np.array([0.0, np.log(3.0)])), [0.0, 0.75 * np.log(3.0)])
