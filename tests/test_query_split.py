"""The arithmetic of the bf16 cached attention's query: a bf16 number as two
e4m3 numbers, the low one's scale 2^-4 of the high one's.  Every significand of
the largest value of a row's 64 channels against every significand and exponent
below it (the sign and the common exponent change nothing)."""
import numpy as np

from oracle import cache as C

SIGNIFICANDS = 1 + np.arange(128) / 128


def split(x, s):
    hi = C.VALUES[C.codes(x / 2.0 ** s)] * 2.0 ** s
    return hi, C.VALUES[C.codes((x - hi) / 2.0 ** (s - 4))] * 2.0 ** (s - 4)


def test_two_parts_hold_a_bf16_value():
    worst = inexact = 0.0
    for top in SIGNIFICANDS:
        s = C.scale_byte([top]) - 127   # smallest power of two with top <= 448 of it
        for k in range(40):
            x = SIGNIFICANDS * 2.0 ** -k
            x = x[x <= top]
            hi, lo = split(x, s)
            assert (np.abs(x - hi) <= np.maximum(x * 2.0 ** -4, 2.0 ** (s - 10))).all(), "a 4-bit rounding"
            off = np.abs(x - (hi + lo))
            worst = max(worst, (off / top).max())
            inexact = max(inexact, (x[off > 0] / top).max(initial=0.0))
    assert 2.0 ** -13.9 < inexact <= 2.0 ** -13.8, "values below 2^-13.8 of the largest may lose bits"
    assert 2.0 ** -21.9 < worst <= 2.0 ** -21.8, "by at most 2^-21.8 of the largest"


def test_one_part_does_not():
    """What a lost low part costs: a 4-bit rounding, 2^-4 of a value."""
    hi, lo = split(SIGNIFICANDS, C.scale_byte([SIGNIFICANDS[-1]]) - 127)
    assert np.abs(SIGNIFICANDS - hi).max() > 2.0 ** -5 and np.array_equal(hi + lo, SIGNIFICANDS)
