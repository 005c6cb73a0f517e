"""The bf16 cached attention's scores are fp32 sums of exact products: the query
goes to the matrix instruction as two e4m3 parts, and the softmax's scale is
applied to the fp32 score.  Outputs against the oracle within the roundings that
are left: of the probabilities and of the result to bf16 (2^-8 each)."""
import numpy as np
import pytest

from gpu_util import log, require_gpu
from oracle import cache as C
from test_gpu_cache import BF16, BF16_HALF, _attend, _bits, _case
from test_gpu_cache_softmax import SIZES, _pages

pytestmark = pytest.mark.gpu


def _tol(q, K, V, p, o, scale):
    """Scores: 2 dim products summed in fp32 (each addition off by at most a step of
    the sum of the magnitudes, truncated sums included), the query's parts off by
    at most 2^-21.8 of the row's largest value, the scale and the exponent by two
    steps of the score; a score error of d changes p by a factor within e^(2 d).
    Then n fp32 additions in the sum and the output, the exponential's own step,
    p's rounding to bf16 and the result's."""
    n, d = K.shape
    mag = (np.abs(q) @ np.abs(K).T).max(1) * abs(scale)
    split = 2.0 ** -21.8 * np.abs(q).max(1) * np.abs(K).sum(1).max() * abs(scale)
    e = (2 * d + 4) * 2.0 ** -23 * mag + split + 2.0 ** -22
    return (p @ np.abs(V)) * (np.expm1(2 * e)[:, None] + BF16_HALF * (1 + BF16_HALF) + (2 * n + 16) * 2.0 ** -23) \
        + np.abs(o) * BF16_HALF + 1e-30


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv_heads,group,qlens,klens,std", [
    (1, 1, [20], [200], 1.0), (2, 1, [300, 1, 70], [200, 33, 64], 1.0), (1, 1, [20], [5000], 1.0), (1, 1, [300], [5000], 1.0),
    (2, 5, [3, 1], [700, 90], 1.0), (8, 5, [260, 300], [129, 512], 1.0), (1, 1, [300], [200], 0.1), (1, 1, [20, 7], [1, 31], 1.0),
    (3, 2, [40, 9], [64, 1000], 3.0)])
def test_only_the_two_roundings_are_left(dim, kv_heads, group, qlens, klens, std):
    B, cache, q, cu, H = _case(BF16, dim, 64, kv_heads, group, qlens, klens, seed=31, std=std)
    o = _attend(B, cache, q, cu, H).double().cpu().numpy()
    x = q.double().cpu().numpy()
    parts = [t[0].cpu().numpy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    table, worst = cache.table.cpu().numpy(), 0.0
    for r, n in enumerate(klens):
        rows = np.unique(np.linspace(cu[r], cu[r + 1] - 1, 60).astype(int))
        for h in range(kv_heads):
            K, V, there = C.gather(*parts, table[r], n, h)
            for j in range(h * group, (h + 1) * group):
                cols = slice(j * dim, (j + 1) * dim)
                want, p = C.attention(x[rows, cols], K, V, there, dim ** -0.5)
                share = np.abs(o[rows, cols] - want) / _tol(x[rows, cols], K, V, p, want, dim ** -0.5)
                worst = max(worst, share.max())
    log(f"  error {worst:.3f} of the tolerance")
    assert worst <= 1


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows,tokens", SIZES)
def test_the_low_part_decides(dim, rows, tokens):
    """Queries whose high parts are the same and take no part in any score.  A
    channel is 16 + u or -(16 + u), u a multiple of 1/8 below 1: high part 16, low
    part u.  The signs alternate and each pair of channels has one key value (1 or
    2, of either sign), so a score is the sum of key x (u - u') over the pairs:
    multiples of 1/8 up to 2^12, exact in fp32 in any order."""
    B = require_gpu()
    log(f"case low parts dim {dim} rows {rows} tokens {tokens}")
    rng = np.random.default_rng(dim + rows)
    pairs = rng.choice([-2.0, -1.0, 1.0, 2.0], (tokens, dim // 2))
    K, V = pairs.repeat(2, 1), C.VALUES[C.codes(rng.standard_normal((tokens, dim)))]
    m = -(-tokens // 32)
    cache = _pages(B, C.codes(K), C.codes(V), np.full(m, 127), np.full(m, 127))
    sign, u = np.where(np.arange(dim) % 2, -1.0, 1.0), rng.integers(0, 8, (rows, dim)) / 8
    q, x = _bits(sign * (16 + u), BF16)
    scale, there = 0.5, np.ones(tokens, bool)
    want, p = C.attention(x, K, V, there, scale)
    # the scale and the exponent: two steps of the score; the sums, the exponential and two roundings as in _tol
    e = 2.0 ** -22 * (1 + np.abs(x @ K.T).max() * scale)
    tol = (p @ np.abs(V)) * (np.expm1(2 * e) + BF16_HALF * (1 + BF16_HALF) + (2 * tokens + 16) * 2.0 ** -23) \
        + np.abs(want) * BF16_HALF
    # a low part that is lost, or of half or twice its size, is far outside
    for wrong in (0.0, 0.5, 2.0):
        other = C.attention(sign * (16 + wrong * u), K, V, there, scale)[0]
        assert ((np.abs(other - want) > 4 * tol).mean(1) > 0.25).mean() > 0.9, wrong
    got = _attend(B, cache, q, [0, rows], 1, scale).double().cpu().numpy()
    log(f"  error {(np.abs(got - want) / tol).max():.3f} of the tolerance")
    assert (np.abs(got - want) <= tol).all()
