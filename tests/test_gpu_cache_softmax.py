"""The cached attention's softmax where its references and sums leave the
ordinary range: scores of 2^33."""
import numpy as np
import pytest
import torch

from gpu_util import log, require_gpu
from oracle import cache as C
from test_gpu_cache import BF16, BF16_HALF, TYPES, _attend, _bits, _fill_real, _request_pages

pytestmark = pytest.mark.gpu
# one short request in whole items or one long one in shares of its tokens, for the
# kernel of few rows (20) and that of many (300)
SIZES = [(20, 200), (300, 200), (20, 5000), (300, 5000)]


def _tokens(cache, n):
    parts = [t[0].cpu().numpy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    K, V, there = C.gather(*parts, cache.table.cpu().numpy()[0], n, 0)
    assert there.all()
    return K, V


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("rows,tokens", SIZES)
@pytest.mark.parametrize("octave", [12, 20, 26, 31, 33, 60, -33])
def test_scores_of_any_size(dtype, dim, rows, tokens, octave):
    """Scaled scores of about 2^octave (log2 units; the octave's sign is the
    scale's): the output is the value of the largest one.  A reference rounded to
    fp32 is off by up to half a step of the score, 2^8 at 2^33."""
    B = require_gpu()
    log(f"case scores of 2^{octave} {dtype} dim {dim} rows {rows} tokens {tokens}")
    rng = np.random.default_rng(octave + 100)
    cache = B.KvCache.empty(-(-tokens // 64) + 1, 1, dim, 64, 1, -(-tokens // 64))
    _fill_real(cache, rng)
    _request_pages(cache, rng, [tokens])
    q, x = _bits(rng.standard_normal((rows, dim)), dtype)
    K, V = _tokens(cache, tokens)
    s = x @ K.T
    scale = float(np.sign(octave) * 2.0 ** abs(octave) / np.log2(np.e) / np.median(np.abs(s).max(1)))
    o = _attend(B, cache, q, [0, rows], 1, scale)
    got = o.double().cpu().numpy()
    s *= scale
    top = np.sort(s, 1)
    # 2 dim sums of fp32 numbers, each off by at most a step of their largest sum, in both scores, and the scaling
    off = 2 * (2 * dim + 4) * 2.0 ** -23 * (np.abs(x) @ np.abs(K).T).max(1) * abs(scale)
    clear = top[:, -1] - top[:, -2] > 40 + off
    assert clear.sum() >= len(x) // 4, "the case is not what it should be"
    assert np.isfinite(got).all()
    want = V[s.argmax(1)]
    # other probabilities are below e^-40; this one's and the result's rounding are left
    half = BF16_HALF if dtype == BF16 else 2.0 ** -20
    bad = (np.abs(got - want)[clear] > 2 * half * np.abs(want)[clear] + 1e-8).any(1)
    assert not bad.any(), f"{bad.sum()} of {len(bad)} rows"
