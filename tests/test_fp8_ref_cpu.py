"""The tests' own 8-bit arithmetic against values worked by hand."""
import numpy as np
import pytest

import fp8_ref as R


def test_codes_round_to_nearest_even():
    for v, code in ((0.0, 0), (448.0, 126), (1.0, 56), (1.0625, 56), (1.1875, 58), (2.0 ** -9, 1), (2.0 ** -10, 0),
                    (1.5 * 2.0 ** -9, 2), (2.0 ** -6, 8), (-1.0, 56 | 128)):
        assert R.e4m3_code(np.array([v]))[0] == code, v


@pytest.mark.parametrize("amax,s", [(448.0, 127), (np.nextafter(448.0, 500), 128), (1.75, 119), (1.7501, 120), (0.0, 0),
                                    (1e-45, 0), (3.4e38, 247), (np.inf, 255), (np.nan, 255)])
def test_scale_bytes(amax, s):
    assert R.scale_byte(amax) == s


def test_every_code_comes_back():
    c = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    assert np.array_equal(R.e4m3_code(R.e4m3_value(c)), c)
