"""The 4-bit cache's scale is max / 7 rounded once, and a code the exact quotient's rounding, for every float16 significand."""

from fractions import Fraction

import numpy as np
import pytest

from oracle import attention_oracle as A

TOPS = np.arange(1024, 2048).astype(np.float32)  # every significand of 11 bits


def heads(channels):
    """[1024, channels]: the largest entry, then odd multiples of its fourteenth part (rounded to float16, ties where that is exact)."""
    x = np.zeros((len(TOPS), channels), np.float16)
    x[:, 0] = TOPS
    for i, odd in enumerate((1, 3, 5, 7, 9, 11, 13)):
        x[:, 1 + i] = (TOPS.astype(np.float64) * odd / 14).astype(np.float16)
        x[:, 8 + i] = -x[:, 1 + i]
    return x


@pytest.mark.parametrize("size", [1.0, 2.0 ** -20, 2.0 ** 5])
def test_scale_and_codes_of_the_oracle_are_the_exact_ones(size):
    x = heads(64).astype(np.float32) * np.float32(size)
    codes, d = A.quantize_heads(x, False)
    for r in range(len(x)):
        want = Fraction(float(x[r, 0])) / 7
        assert abs(Fraction(float(d[r])) - want) <= Fraction(float(np.spacing(d[r]))) / 2
        for c in range(15):
            assert codes[r, c] == round(Fraction(float(x[r, c])) / Fraction(float(d[r])))  # (half to even)
