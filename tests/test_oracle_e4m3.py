"""Pins of the 8-bit cache oracle: the format's numbers, rounding and scales."""
import numpy as np
import pytest
import torch

from oracle import e4m3


def test_numbers_are_the_formats():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(e4m3.NUMBERS, codes)
    assert e4m3.NUMBERS[-1] == 448 and e4m3.NUMBERS[1] == 2.0 ** -9


def test_nearest_on_every_number_midpoint_and_side():
    n = e4m3.NUMBERS
    mid = (n[1:] + n[:-1]) / 2
    even = np.where(np.arange(126) % 2 == 0, n[:-1], n[1:])
    np.testing.assert_array_equal(e4m3.nearest(n), n)
    np.testing.assert_array_equal(e4m3.nearest(-n), -n)
    np.testing.assert_array_equal(e4m3.nearest(mid), even)
    np.testing.assert_array_equal(e4m3.nearest(mid * (1 + 1e-12)), n[1:])
    np.testing.assert_array_equal(e4m3.nearest(mid * (1 - 1e-12)), n[:-1])
    np.testing.assert_array_equal(e4m3.nearest(mid), torch.tensor(mid).float().to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("top,e", [(448.0, 0), (np.nextafter(448.0, 449), 1), (224.0, -1), (1.0, -8), (1.75, -8),
                                   (1.76, -7), (0.0, -117), (2.0 ** -133, -117), (448 * 2.0 ** -117, -117),
                                   (449 * 2.0 ** -117, -116), (1.9 * 2.0 ** 127, 120)])
def test_scale_exponents(top, e):
    assert e4m3.exponent(np.array(top)) == e
    assert top <= 448 * 2.0 ** e and (e == -117 or top > 448 * 2.0 ** (e - 1))


def test_relative_error_is_half_a_step_and_tokens_that_are_not_finite_are_nan():
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((5, 3, 64)), rng.standard_normal((5, 3, 64)) * 1e3
    sk, sv = e4m3.store_kv(k, v)
    for x, s in ((k, sk), (v, sv)):
        f = 2.0 ** e4m3.exponent(np.abs(x).max(-1, keepdims=True))
        assert (np.abs(s - x) <= np.maximum(np.abs(x) * 2.0 ** -4, f * 2.0 ** -10)).all()
    k[1, 2, 5], v[3, 0, 0] = np.inf, np.nan
    sk2, sv2 = e4m3.store_kv(k, v)
    for t, h in ((1, 2), (3, 0)):
        assert np.isnan(sk2[t, h]).all() and np.isnan(sv2[t, h]).all()
    keep = np.ones((5, 3), bool)
    keep[1, 2] = keep[3, 0] = False
    np.testing.assert_array_equal(sk2[keep], sk[keep])
    np.testing.assert_array_equal(sv2[keep], sv[keep])
