"""The oracle of the Linears on 8-bit integers, against what does not use it."""
from fractions import Fraction

import numpy as np

from oracle import rows_i8 as R


def _nearest_even(q: Fraction) -> int:
    low = q.numerator // q.denominator
    rest = q - low
    if rest == Fraction(1, 2):
        return low + low % 2
    return low + (rest > Fraction(1, 2))


def test_codes_are_the_nearest_whole_steps_in_exact_arithmetic():
    """Rows of 8-bit significands, whose values are often exactly between two codes."""
    rng = np.random.default_rng(5)
    y = rng.integers(-255, 256, (40, 96)).astype(np.float64) * 2.0 ** rng.integers(-4, 3, (40, 96))
    y[:10] = rng.integers(-254, 255, (10, 96))
    y[:10, 7] = 254                      # 127 y / m = y / 2
    codes, scales = R.quantize(y)
    ties = 0
    for r in range(len(y)):
        m = max(abs(Fraction(v)) for v in y[r])
        for v, c in zip(y[r], codes[r]):
            q = 127 * Fraction(v) / m
            ties += q.denominator == 2
            assert c == _nearest_even(q)
        assert scales[r] == float(m) / 127
    assert ties > 300


def test_a_code_is_within_half_a_step_and_the_largest_is_127():
    y = np.random.default_rng(6).standard_normal((30, 77)) * np.logspace(-27, 30, 30)[:, None]   # above 127 x 2^-100 = 1e-28
    codes, scales = R.quantize(y)
    # y - c s is a difference of numbers up to 127 s, each rounded to 2^-53
    assert (np.abs(y - codes * scales[:, None]) <= scales[:, None] * (0.5 + 256 * 2.0 ** -53)).all()
    assert (np.abs(codes).max(1) == 127).all()


def test_rows_without_values_and_rows_that_are_not_finite():
    y = np.zeros((4, 16))
    y[1, 3], y[2, 0], y[3, 5] = np.inf, np.nan, 2.0 ** -120
    codes, scales = R.quantize(y)
    assert (codes == 0).all()
    assert scales[0] == scales[3] == 2.0 ** -100 and np.isnan(scales[1]) and np.isnan(scales[2])


def test_modulated_rows_have_the_moments_of_their_vectors():
    rng = np.random.default_rng(7)
    x, cu = rng.standard_normal((9, 4096)) * 3 + 5, [0, 4, 4, 9]
    shift, scale = rng.standard_normal((3, 1)) * np.ones(4096), rng.standard_normal((3, 1)) * np.ones(4096)
    y = R.modulate(x, shift, scale, cu, 1e-12)
    for rows, r in ((slice(0, 4), 0), (slice(4, 9), 2)):
        assert np.allclose(y[rows].mean(1), shift[r, 0], atol=1e-12)
        assert np.allclose(y[rows].std(1), abs(1 + scale[r, 0]), atol=1e-12)


def test_rms_rows_have_unit_mean_square():
    x = np.random.default_rng(8).standard_normal((5, 1024)) * 7
    assert np.allclose((R.rms(x, np.ones(1024), 0.0) ** 2).mean(1), 1)
    assert np.allclose(R.rms(x, np.full(1024, 3.0), 1e12), x * 3e-6, rtol=1e-7)


def test_product_against_python_integers():
    rng = np.random.default_rng(9)
    a, w = rng.integers(-128, 128, (3, 4096)).astype(np.int8), rng.integers(-128, 128, (4, 4096)).astype(np.int8)
    a[0], w[0] = -128, -128
    want = [[sum(int(x) * int(y) for x, y in zip(ra, rw)) for rw in w] for ra in a]
    assert (R.sums(a, w) == np.array(want)).all()
    sa, sw = np.array([2.0, 0.5, 1.0]), np.array([1.0, 4.0, 0.25, 3.0])
    z = np.array(want) * sa[:, None] * sw
    res, gate = rng.standard_normal((3, 4)), rng.standard_normal((2, 4))
    assert (R.linear(a, sa, w, sw) == z).all()
    got = R.linear(a, sa, w, sw, np.ones(4), "gated", res, gate, [0, 1, 3])
    assert np.allclose(got[0], res[0] + gate[0] * (z[0] + 1)) and np.allclose(got[2], res[2] + gate[1] * (z[2] + 1))
    assert np.allclose(R.linear(a, sa, w, sw, None, "residual", res), res + z)
    assert np.allclose(R.gelu_tanh(np.array([-30.0, 0.0, 30.0])), [0, 0, 30])
