"""The cached attention's softmax where its references and sums leave the
ordinary range: scores of 2^33, values whose products with an unfinished
probability pass fp32, scores of minus infinity."""
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


def _pages(B, k, v, ks, vs, page=32):
    """A cache of one request and head with these codes [tokens, channels] and scale bytes per page."""
    n, d = k.shape
    m = -(-n // page)
    c = B.KvCache.empty(m, 1, d, page, 1, m)
    for pool, codes, place in ((c.k, k, C.k_place), (c.v, v, C.v_place)):
        x = np.full(tuple(pool.shape[3:]), 0x7F, np.uint8)
        x = np.broadcast_to(x, (m,) + x.shape).copy()
        for p in range(m):
            rows = codes[p * page:(p + 1) * page]
            t, ch = np.meshgrid(np.arange(len(rows)), np.arange(d), indexing="ij")
            x[p][place(t, ch)] = rows
        pool[0, :, 0] = torch.from_numpy(x).cuda()
    c.k_scale[0, :, 0] = torch.from_numpy(np.asarray(ks, np.uint8)).cuda()
    c.v_scale[0, :, 0] = torch.from_numpy(np.asarray(vs, np.uint8)).cuda()
    c.table.copy_(torch.arange(m, dtype=torch.int32).view(1, m))
    c.lens.fill_(n)
    return c


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


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("rows,tokens", SIZES)
@pytest.mark.parametrize("byte,code", [(197, 1.5), (175, 448.0), (176, -448.0), (247, -192.0)])
def test_large_values(dtype, dim, rows, tokens, byte, code):
    """One token's score lies 60 octaves over the others', below the 2^64 at which
    a row's sum alone would show it, and its value times 2^60 passes fp32."""
    B = require_gpu()
    log(f"case value {code} x 2^{byte - 127} {dtype} dim {dim} rows {rows} tokens {tokens}")
    m, far = -(-tokens // 32), tokens - 70
    k, v = np.zeros((tokens, dim), np.uint8), np.zeros((tokens, dim), np.uint8)
    k[far, 0] = C.codes(60.0)
    v[far] = C.codes(code * (1 - 0.5 * (np.arange(dim) % 2)))   # the code and half of it in turn
    vs = np.full(m, 120)
    vs[far // 32] = byte
    cache = _pages(B, k, v, np.full(m, 127), vs)
    q, _ = _bits(np.eye(1, dim).repeat(rows, 0), dtype)
    o = _attend(B, cache, q, [0, rows], 1, float(np.log(2)))   # a score of 60 is 2^60
    got = o.double().cpu().numpy()
    want = C.VALUES[v[far]] * 2.0 ** (byte - 127)
    half = BF16_HALF if dtype == BF16 else 2.0 ** -20
    assert (np.abs(got - want) <= 2 * half * np.abs(want)).all(), (got[0, :2], want[:2])


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("rows,tokens", SIZES)
@pytest.mark.parametrize("where", ["first", "last"])
def test_scores_of_minus_infinity(dtype, dim, rows, tokens, where):
    """Tokens whose score is below fp32's range have no weight, in front of the
    others or behind them, in some rows of a call and not in others."""
    B = require_gpu()
    log(f"case scores of minus infinity {where} {dtype} dim {dim} rows {rows} tokens {tokens}")
    rng = np.random.default_rng(3)
    m, n = -(-tokens // 32), tokens // 2 // 32 * 32
    k = np.zeros((tokens, dim), np.uint8)
    low = np.arange(tokens) < n if where == "first" else np.arange(tokens) >= n
    k[low, 0] = C.codes(32.0)
    v = C.codes(rng.standard_normal((tokens, dim)))
    cache = _pages(B, k, v, np.full(m, 152), np.full(m, 127))   # 2^5 * 2^25
    x = np.zeros((rows, dim))
    x[:, 0] = np.where(np.arange(rows) % 3, -2.0 ** 100, 0.0)   # powers of two: the whole product overflows, not a part of it
    q, _ = _bits(x, dtype)
    got = _attend(B, cache, q, [0, rows], 1).double().cpu().numpy()
    V = C.VALUES[v]
    for r in range(rows):
        use = V[~low] if r % 3 else V
        want = use.mean(0)
        # equal scores: bf16 probabilities of exactly 1, fp32 sums of the values, the result's rounding
        tol = (BF16_HALF if dtype == BF16 else 2.0 ** -23) * np.abs(want) + (len(use) + 16) * 2.0 ** -24 * np.abs(use).mean(0)
        assert (np.abs(got[r] - want) <= tol).all(), (r, got[r, :3], want[:3])
