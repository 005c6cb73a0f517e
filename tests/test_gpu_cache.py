"""The paged 8-bit key/value cache on the GPU against its oracle.

Tables, slot maps, codes and scale bytes are equal to the oracle's.  Attention
tolerances come from the roundings that the kernels make, relative to the
oracle's own probabilities p and values V (``_attention_tol``)."""
import numpy as np
import pytest
import torch

import synth
from gpu_util import dev, host, log, require_gpu
from oracle import cache as C

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
BF16_HALF = 2.0 ** -8   # a rounding to bf16 (8 significant bits) is off by at most this much of the value


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _u8(a):
    return a.cpu().numpy()


# ------------------------------------------------------------------- tables


def _tables(page, width, before, added, n_free, per=0, n_rows=None, rows=None, null_before=False, extra=3):
    """One call against the oracle; the table is full of other numbers before it."""
    B = require_gpu()
    n = len(added)
    rows = rows or n
    rng = np.random.default_rng(page + n)
    n_rows = (n * per if per else sum(max(a, 0) for a in added)) if n_rows is None else n_rows
    cache = B.KvCache.empty(1, 1, 64, page, rows, width)
    start = rng.integers(100, 10 ** 6, (rows, width)).astype(np.int32)
    cache.table.copy_(torch.from_numpy(start))
    cache.lens.fill_(-7)
    free = rng.permutation(10 ** 5)[:n_free].astype(np.int32)
    runs = torch.full((B.cache_run_bound(page, n, n_rows) + extra, 4), -5, dtype=torch.int32, device="cuda")
    counts = _i32([-1] * 4)
    # a stack of free pages whose top is anywhere: no alignment but an integer's
    stack = _i32(np.r_[np.full(n % 4, -9, np.int32), free])[n % 4:]
    B.cache_tables(cache, None if null_before else _i32(before), _i32(added), stack if n_free else None, runs, counts,
                   n_rows, per)
    torch.cuda.synchronize()
    tab, lens, want, cnt = C.tables(page, start, [0] * n if null_before else before, added, free, n_rows, per)
    assert np.array_equal(cache.table.cpu().numpy(), tab)
    assert cache.lens.tolist() == lens + [-7] * (rows - n)
    assert counts.tolist() == cnt
    got = runs.cpu().numpy()
    assert [tuple(x) for x in got[:len(want)].tolist()] == want
    assert (got[len(want):] == 0).all()


@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_tables_vs_oracle(page):
    log(f"case tables page {page}")
    rng = np.random.default_rng(page)
    _tables(page, 4, [0], [77], 9, null_before=True)
    _tables(page, 9, [0], [1], 1)
    _tables(page, 9, [page], [0], 0)                                   # nothing to do, no free page
    _tables(page, 9, [page - 1, page, page + 1], [1, 1, 2 * page], 9)  # up to a page's end, from its start, over two ends
    _tables(page, 40, rng.integers(0, 20 * page, 64), rng.integers(0, 12 * page, 64), 64 * 13, rows=70)
    _tables(page, 40, rng.integers(0, 20 * page, 64), rng.integers(0, 3, 64), 64)      # single tokens
    _tables(page, 40, rng.integers(0, 20 * page, 7), rng.integers(0, 300, 7), 99, per=300)


@pytest.mark.parametrize("page", [32, 128])
def test_tables_refuse_requests(page):
    log(f"case tables refusals page {page}")
    full = 10 * page
    _tables(page, 10, [0, 5, 0, 3], [2 * page, 3, 9 * page, 4], 6)     # the third does not fit, the fourth needs no page
    _tables(page, 10, [0, 0, 0], [page, 3 * page, page], 3)            # nor does a later one that would
    _tables(page, 10, [full - 1, full, full - 2, 0], [1, 1, 3, 9], 5)  # rows of the table end
    _tables(page, 10, [-1, 0, -2 ** 31, 4, full + 9], [3, -4, 5, 6, 0], 5)
    _tables(page, 10, [0, 0, 0], [2 ** 31 - 1, 2 ** 31 - 1, 7], 5, n_rows=50)          # sums past 32 bits
    _tables(page, 10, [2 ** 31 - 1, 0], [2 ** 31 - 1, 7], 5, n_rows=50)
    _tables(page, 10, [0, 0, 0], [30, 30, 30], 5, n_rows=70)           # the last one's rows are not there
    _tables(page, 10, [0, 0, 0], [30, 31, 30], 5, per=30)
    _tables(page, 10, [0, 3], [page, page], 0)


# -------------------------------------------------------------------- store


def _filled(B, rng, n_pages, heads, dim, page, rows, width, blocks=1):
    """A cache whose pages hold other requests' codes, NaN among them."""
    c = B.KvCache.empty(n_pages, heads, dim, page, rows, width, blocks)
    for t in (c.k, c.v):
        t.copy_(torch.from_numpy(rng.integers(0, 256, t.shape).astype(np.uint8)))
    for t in (c.k_scale, c.v_scale):
        t.copy_(torch.from_numpy(rng.integers(118, 124, t.shape).astype(np.uint8)))
    return c


def _bits(x, dtype):
    """fp32 numbers as a device tensor of dtype, and the numbers it holds."""
    t = torch.from_numpy(np.asarray(x, np.float32)).to(dtype)
    return t.cuda(), t.double().numpy()


def _store_oracle(cache0, block, k, v, runs, heads, dim, page):
    out = [t[block].copy() for t in cache0]
    for p, row, off, n in runs:
        if n <= 0 or not (0 <= p < out[0].shape[0] and 0 <= off and off + n <= page and 0 <= row and row + n <= len(k)):
            continue
        for i, (x, place) in enumerate(((k, C.k_place), (v, C.v_place))):
            for h in range(heads):
                out[i][p, h], out[2 + i][p, h] = C.store(out[i][p, h], out[2 + i][p, h], x[row:row + n, h * dim:(h + 1) * dim],
                                                         off, place)
    return out


def _store(B, cache, k, v, runs, block, ks=None, vs=None):
    """Stores and compares the whole pools with the oracle's."""
    heads, dim, page = cache.c.n_kv_heads, cache.c.head_dim, cache.c.page_tokens
    before = [_u8(t) for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    B.cache_store(cache, k, v, _i32(runs), block=block)
    torch.cuda.synchronize()
    want = _store_oracle(before, block, k.double().cpu().numpy(), v.double().cpu().numpy(), runs, heads, dim, page)
    for name, t, w, b in zip(("k", "v", "k_scale", "v_scale"), (cache.k, cache.v, cache.k_scale, cache.v_scale), want, before):
        b[block] = w
        got = _u8(t)
        if name in "kv":   # by value: a rescaled negative may be either zero, a NaN either NaN
            assert np.array_equal(C.VALUES[got], C.VALUES[b], equal_nan=True), name
        else:
            assert np.array_equal(got, b), name


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_store_vs_oracle(dtype, dim, page):
    B = require_gpu()
    log(f"case store {dtype} dim {dim} page {page}")
    rng = np.random.default_rng(dim + page)
    heads = 3
    for runs in ([(4, 0, 0, page)], [(1, 0, 0, 1), (3, 1, 0, page - 1), (0, page, 5, 7), (2, page + 7, page - 1, 1), (0, 0, 0, 0)],
                 [(0, 0, page // 2, page // 2), (4, page // 2, 16, 1), (1, page // 2 + 1, 17, 3)]):
        n = max(r[1] + r[3] for r in runs)
        cache = _filled(B, rng, 5, heads, dim, page, 1, 1, blocks=2)
        # rows of [k | v] and a gap, of magnitudes that differ from token to token
        x = rng.standard_normal((n, 2 * heads * dim + 16)) * 2.0 ** rng.integers(-6, 7, (n, 1))
        kv, _ = _bits(x, dtype)
        _store(B, cache, kv[:, :heads * dim], kv[:, heads * dim:2 * heads * dim], runs, 1)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_store_values_at_borders(dtype):
    B = require_gpu()
    log(f"case store borders {dtype}")
    rng = np.random.default_rng(4)
    mid = (C.VALUES[1:127] + C.VALUES[:126]) / 2
    rows = [np.r_[448.0, 448.0, mid], np.r_[464.0, 464.0, -mid], np.zeros(128), np.full(128, -0.0), np.full(128, 2.0 ** -120),
            np.r_[np.inf, -np.inf, np.nan, np.ones(125)], np.full(128, np.nan), np.r_[3.38e38, rng.standard_normal(127)],
            np.r_[449.0, 447.9, np.ones(126)], np.r_[2.0 ** -100 * 448, np.full(127, 2.0 ** -109)]]
    for x in rows:
        for off in (0, 9):
            cache = _filled(B, rng, 2, 1, 128, 32, 1, 1)
            t, _ = _bits(np.stack([x, x[::-1]]), dtype)
            _store(B, cache, t, t.clone(), [(1, 0, off, 2)], 0)


def test_store_token_by_token():
    """A page filled one token at a time holds what the oracle's does, whose
    scale grows along the way."""
    B = require_gpu()
    rng = np.random.default_rng(5)
    cache = _filled(B, rng, 2, 2, 64, 32, 1, 1)
    for t in range(32):
        log(f"case store token {t}") if t % 8 == 0 else None
        x, _ = _bits(rng.standard_normal((2, 128)) * 1.3 ** t, BF16)
        _store(B, cache, x[:1], x[1:], [(1, 0, t, 1)], 0)


def test_store_skips_bad_entries():
    B = require_gpu()
    log("case store bad entries")
    rng = np.random.default_rng(6)
    cache = _filled(B, rng, 3, 2, 64, 64, 1, 1)
    x, _ = _bits(rng.standard_normal((10, 128)), BF16)
    big = 2 ** 31 - 1
    _store(B, cache, x, x.clone(), [(-1, 0, 0, 4), (3, 0, 0, 4), (big, 0, 0, 4), (0, -1, 0, 4), (0, 7, 0, 4), (0, big, 0, 4),
                                    (0, 0, -1, 4), (0, 0, 61, 4), (0, 0, big, 4), (0, 0, 0, -4), (0, 0, 0, big), (0, 0, big, big),
                                    (1, 2, 3, 4)], 0)


# ---------------------------------------------------------------- attention


def _attention_tol(q, K, V, p, o, scale, dtype):
    """bf16: the scaled query is rounded (each channel by at most 2^-8 of its
    value, independently, so the score's error has a standard deviation of at
    most 2^-8 / sqrt(3) * scale * sqrt(sum q^2 k^2); 8 of them are allowed), the
    probabilities too (2^-8 of each), and the result (2^-8).  A score error of d
    changes p by a factor within e^(2 d).
    fp32: sums of n terms, n 2^-24 of the sum of their magnitudes."""
    if dtype == BF16:
        var = (q * q) @ (K * K).T if len(K) else np.zeros((len(q), 1))
        d = 8 * BF16_HALF / np.sqrt(3) * abs(scale) * np.sqrt(var.max(1)) + 1e-5
        return (p @ np.abs(V)) * (np.expm1(2 * d)[:, None] + BF16_HALF) + np.abs(o) * BF16_HALF + 1e-30
    mag = (np.abs(q) @ np.abs(K).T if len(K) else np.zeros((len(q), 1))).max(1) * abs(scale)
    d = (q.shape[1] + 4) * 2.0 ** -24 * mag
    return (p @ np.abs(V)) * (np.expm1(2 * d)[:, None] + (len(K) + 16) * 2.0 ** -24) + 1e-30


def _fill_real(cache, rng, std=1.0):
    """Pages of normal values (no NaN) with scales around 2^-8."""
    for t in (cache.k, cache.v):
        x = torch.randn(t.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30))))
        t.copy_((x * 110 * std).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    for t in (cache.k_scale, cache.v_scale):
        t.copy_(torch.from_numpy(rng.integers(118, 122, t.shape).astype(np.uint8)))


def _request_pages(cache, rng, lens):
    """Distinct pages in random order; entries behind a request's pages are out of range."""
    P, width = cache.c.page_tokens, cache.c.max_pages
    order = rng.permutation(cache.c.n_pages)
    table = np.full((cache.c.table_rows, width), 2 ** 31 - 1, np.int64)
    at = 0
    for r, n in enumerate(lens):
        k = min(-(-max(n, 0) // P), width)
        table[r, :k] = order[at:at + k]
        at += k
    cache.table.copy_(torch.from_numpy(table.astype(np.int32)))
    cache.lens.copy_(_i32(list(lens) + [0] * (cache.c.table_rows - len(lens))))


def _nan_behind(cache, lens):
    """NaN codes in every place of the last pages behind the requests' tokens."""
    P = cache.c.page_tokens
    table = cache.table.cpu().numpy()
    for r, n in enumerate(lens):
        if n <= 0 or n % P == 0:
            continue
        p = int(table[r, n // P])
        for t in range(n % P, P):
            g, u = t // 32, t % 32
            cache.k[:, p, :, g, :, u, :] = 0x7F
            cache.v[:, p, :, g, u // 4 % 2, :, u // 8 * 4 + u % 4] = 0xFF


def _check_attention(cache, q, o, cu, n_heads, scale=None, block=0, max_len=0, rows=None):
    """Rows of o against the oracle; ``rows``: that many of each request (all by default)."""
    dim, G, dtype = cache.c.head_dim, n_heads // cache.c.n_kv_heads, q.dtype
    parts = [t[block].cpu().numpy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    table, lens = cache.table.cpu().numpy(), cache.lens.tolist()
    scale = dim ** -0.5 if scale is None else scale
    cap = min(cache.c.max_pages * cache.c.page_tokens, max_len or 2 ** 31)
    worst = 0.0
    for r in range(len(cu) - 1):
        n = cu[r + 1] - cu[r]
        if n == 0:
            continue
        idx = np.arange(n) if rows is None or n <= rows else np.unique(np.r_[0, n - 1, np.linspace(0, n - 1, rows).astype(int)])
        qr = q[cu[r]:cu[r + 1]][idx].double().cpu().numpy()
        got = o[cu[r]:cu[r + 1]][idx].double().cpu().numpy()
        for h in range(cache.c.n_kv_heads):
            K, V, there = C.gather(*parts, table[r], min(max(lens[r], 0), cap), h)
            for j in range(h * G, (h + 1) * G):
                x = qr[:, j * dim:(j + 1) * dim]
                want, p = C.attention(x, K, V, there, scale)
                g = got[:, j * dim:(j + 1) * dim]
                assert np.isfinite(g).all(), (r, j)
                if not there.any():
                    assert (g == 0).all()
                    continue
                tol = _attention_tol(x, K[there], V[there], p, want, scale, dtype)
                worst = max(worst, (np.abs(g - want) / tol).max())
                assert (np.abs(g - want) <= tol).all(), (r, j, np.abs(g - want).max(), tol.max())
    log(f"  error {worst:.3f} of the tolerance")


def _attend(B, cache, q, cu, n_heads, scale=None, block=0, max_len=0, o=None, stream=None):
    o = torch.full_like(q, float("nan")) if o is None else o
    n = B.attention_cached_workspace_size(cache, cu, n_heads, q.dtype, max_len)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None
    B.attention_cached(cache, q, o, cu, n_heads, ws, block, max_len, scale, stream)
    return o


def _case(dtype, dim, page, kv_heads, group, qlens, klens, seed, std=1.0, width=None, **kw):
    B = require_gpu()
    log(f"case attention {dtype} dim {dim} page {page} heads {kv_heads}x{group} q {qlens} k {klens} {kw}")
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in klens]
    cache = B.KvCache.empty(sum(need) + 2, kv_heads, dim, page, len(klens), width or max(max(need), 1))
    _fill_real(cache, rng)
    _request_pages(cache, rng, klens)
    _nan_behind(cache, klens)
    cu = [0] + np.cumsum(qlens).tolist()
    H = kv_heads * group
    q, _ = _bits(rng.standard_normal((cu[-1], H * dim)) * std, dtype)
    return B, cache, q, cu, H


TYPES = [(BF16, 128), (BF16, 64), (F32, 64), (F32, 128)]


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("page", [32, 64, 128, 256])
@pytest.mark.parametrize("qlens,klens", [
    ([1], [1]), ([40], [33]), ([5, 3, 1], [64, 0, 31]), ([0, 70, 0, 1], [5, 130, 3, 257]), ([129, 128, 127], [63, 64, 65]),
    ([32, 7], [1, 511])])
def test_attention_vs_oracle(dtype, dim, page, qlens, klens):
    B, cache, q, cu, H = _case(dtype, dim, page, 2, 1, qlens, klens, seed=dim + page)
    _check_attention(cache, q, _attend(B, cache, q, cu, H), cu, H)


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("kv_heads,group,qlens,klens", [
    (1, 5, [1, 2, 0], [200, 77, 9]), (3, 2, [16, 5], [100, 300]), (2, 33, [1], [90]), (2, 5, [100, 3], [70, 400]), (40, 1, [1], [512])])
def test_attention_head_groups(dtype, dim, kv_heads, group, qlens, klens):
    B, cache, q, cu, H = _case(dtype, dim, 64, kv_heads, group, qlens, klens, seed=kv_heads * group)
    _check_attention(cache, q, _attend(B, cache, q, cu, H), cu, H)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv_heads,group,qlens,klens", [
    (40, 1, [1001, 0, 333, 450], [512, 9, 0, 77]), (24, 1, [33, 2000, 1000], [1, 300, 65]), (8, 5, [1500, 31, 300], [18, 512, 129]),
    (1, 40, [1664, 3], [500, 64])])
@pytest.mark.parametrize("page", [32, 256])
def test_attention_many_rows_on_prompts(dim, kv_heads, group, qlens, klens, page):
    """More than 8 blocks of 32 rows per compute unit on prompts up to 512
    tokens (that bound given where the table is wider), missing pages, a bound
    that ends inside a tile, and the same bits from every call."""
    B, cache, q, cu, H = _case(BF16, dim, page, kv_heads, group, qlens, klens, seed=20, width=4096 // page)
    rows = 5 if kv_heads * group > 8 else 40
    first = _attend(B, cache, q, cu, H, max_len=512)
    _check_attention(cache, q, first, cu, H, max_len=512, rows=rows)
    for _ in range(3):
        assert torch.equal(_attend(B, cache, q, cu, H, max_len=512), first)
    cache.table[1, 0] = -1
    cache.table[0, (klens[0] - 1) // page] = cache.c.n_pages
    _check_attention(cache, q, _attend(B, cache, q, cu, H, max_len=512), cu, H, max_len=512, rows=rows)
    bound = 70   # inside a tile
    _check_attention(cache, q, _attend(B, cache, q, cu, H, max_len=bound), cu, H, max_len=bound, rows=rows)


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("qlens,klens", [([1], [9000]), ([3, 1, 2], [5000, 100, 0]), ([200], [9001]), ([130, 20], [4100, 700])])
def test_attention_divided_tokens(dtype, dim, qlens, klens):
    """Few queries over many tokens: key pieces in the workspace, some of them empty."""
    B, cache, q, cu, H = _case(dtype, dim, 128, 2, 1, qlens, klens, seed=11)
    assert B.attention_cached_workspace_size(cache, cu, H, dtype) > 0
    _check_attention(cache, q, _attend(B, cache, q, cu, H), cu, H, rows=40)


@pytest.mark.parametrize("qlens", [[2], [50]])
def test_attention_long_history(qlens):
    """Past the groups that are looked up at once (32,768 tokens), divided or not."""
    B, cache, q, cu, H = _case(BF16, 128, 64, 1, 1, qlens, [70001], seed=12)
    _check_attention(cache, q, _attend(B, cache, q, cu, H), cu, H, rows=12)
    many = torch.cat([q] * (-(-128 * 2048 // len(q))))[:128 * 2048].contiguous()   # four rounds of workgroups: not divided
    cu = [0, len(many)]
    assert B.attention_cached_workspace_size(cache, cu, H, BF16) == 0
    _check_attention(cache, many, _attend(B, cache, many, cu, H), cu, H, rows=12)


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("qlens", [[3, 4], [150, 40]])
def test_attention_missing_pages(dtype, dim, qlens):
    """Tokens on pages outside the pool are not there: at the start, inside a
    tile, at the end, all of them."""
    B, cache, q, cu, H = _case(dtype, dim, 32, 2, 1, qlens, [300, 290], seed=13)
    for bad in ([0], [0, 1], [0, 1, 2, 3, 4], [3], [9], [2, 5, 8], list(range(10))):
        log(f"  missing {bad}")
        table = cache.table.clone()
        cache.table[0, bad] = _i32([(-1, -2 ** 31, 2 ** 31 - 1, cache.c.n_pages)[i % 4] for i in range(len(bad))])
        _check_attention(cache, q, _attend(B, cache, q, cu, H), cu, H)
        cache.table.copy_(table)


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("qlens", [[3, 4, 2], [150, 40, 35]])
def test_attention_lengths_and_bound(dtype, dim, qlens):
    """Lengths below 0 and past the table's width, and the call's own bound."""
    B, cache, q, cu, H = _case(dtype, dim, 64, 2, 1, qlens, [256, 200, 256], seed=14)
    cache.lens.copy_(_i32([2 ** 31 - 1, -5, 257]))
    _check_attention(cache, q, _attend(B, cache, q, cu, H), cu, H)
    cache.lens.copy_(_i32([256, 200, 30]))
    for bound in (1, 33, 64, 199, 255, 10 ** 6):
        _check_attention(cache, q, _attend(B, cache, q, cu, H, max_len=bound), cu, H, max_len=bound)


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("qlens", [[9], [90]])
@pytest.mark.parametrize("scale", [0.5, -0.3, 1e-6])
def test_attention_softmax_scale(dtype, dim, qlens, scale):
    B, cache, q, cu, H = _case(dtype, dim, 64, 2, 1, qlens, [150], seed=15, std=0.5)
    _check_attention(cache, q, _attend(B, cache, q, cu, H, scale), cu, H, scale)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("qlens", [[20], [300], [33000]])
@pytest.mark.parametrize("order", ["rising", "falling"])
def test_attention_far_scores(dim, qlens, order):
    """Scores that rise by hundreds of octaves from tile to tile (past the range
    of a probability against the first tile), or fall so: one token's value."""
    B, cache, q, cu, H = _case(BF16, dim, 32, 2, 1, qlens, [320], seed=16, std=3.0)
    ramp = np.arange(10) if order == "rising" else np.arange(10)[::-1]
    table = cache.table.cpu().numpy()[0]
    for i in range(10):
        cache.k_scale[0, int(table[i])] = int(114 + 2 * ramp[i])
    o = _attend(B, cache, q, cu, H)
    # the largest score leads by far more than its rounding: the output is that token's value
    parts = [t[0].cpu().numpy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    for h in range(2):
        K, V, there = C.gather(*parts, table, 320, h)
        x = q[:, h * dim:(h + 1) * dim].double().cpu().numpy()
        s = x @ K.T * dim ** -0.5
        top = np.sort(s, 1)
        clear = top[:, -1] - top[:, -2] > 40 + 2 * BF16_HALF * np.abs(x).sum(1) * np.abs(K).max() * dim ** -0.5   # both scores' rounding
        assert clear.sum() > len(x) // 4, "the case is not what it should be"
        got = o[:, h * dim:(h + 1) * dim].double().cpu().numpy()
        assert np.isfinite(got).all()
        want = V[s.argmax(1)]
        # the other probabilities are below e^-40; this one may be near 1, not 1 (its reference is the maximum of scores
        # summed in another order), and its rounding against its unrounded sum and the result's rounding are left
        assert (np.abs(got - want)[clear] <= 2 * BF16_HALF * np.abs(want)[clear] + 1e-8).all()


def test_attention_strides_blocks_streams():
    """Row strides, a block's pool behind another's, rows of the output's gaps
    left as they were, a stream of the caller's."""
    B = require_gpu()
    rng = np.random.default_rng(17)
    for dtype, qlens in ((BF16, [5, 0, 6]), (BF16, [150, 0, 3]), (F32, [5, 0, 6])):
        log(f"case attention strides {dtype} {qlens}")
        cache = B.KvCache.empty(20, 2, 128, 64, 4, 6, n_blocks=3)
        _fill_real(cache, rng)
        _request_pages(cache, rng, [300, 5, 128])
        cu = [0] + np.cumsum(qlens).tolist()
        q, _ = _bits(rng.standard_normal((cu[-1] + 2, 600)), dtype)
        o = torch.full((cu[-1] + 2, 552), 3.0, dtype=dtype, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        _attend(B, cache, q[:, :512], cu, 4, block=2, o=o[:, :512], stream=s)
        torch.cuda.current_stream().wait_stream(s)
        _check_attention(cache, q[:, :512], o[:, :512], cu, 4, block=2)
        assert (o[:, 512:] == 3).all() and (o[cu[-1]:] == 3).all()


def test_attention_pool_past_32_bits():
    """Pages whose byte offsets pass 2^32."""
    B = require_gpu()
    log("case attention on pages past 4 GiB")
    rng = np.random.default_rng(18)
    cache = B.KvCache.empty(140000, 1, 128, 256, 2, 2)
    near = B.KvCache.empty(4, 1, 128, 256, 2, 2)
    _fill_real(near, rng)
    far = [139999, 131072, 70000, 3]
    for t, f in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), (near.k, near.v, near.k_scale, near.v_scale)):
        t[:, far] = f
    for n in (3, 90):
        cu = [0, n, 2 * n]
        q, _ = _bits(rng.standard_normal((2 * n, 128)), BF16)
        for c, pages in ((cache, far), (near, [0, 1, 2, 3])):
            c.table.copy_(_i32(pages).view(2, 2))
            c.lens.copy_(_i32([512, 300]))
        a, b = _attend(B, cache, q, cu, 1), _attend(B, near, q, cu, 1)
        assert torch.equal(a, b)
        _check_attention(near, q, b, cu, 1)
    x, _ = _bits(rng.standard_normal((256, 128)), BF16)
    B.cache_store(cache, x, x.clone(), _i32([(139999, 0, 0, 256)]))
    B.cache_store(near, x, x.clone(), _i32([(0, 0, 0, 256)]))
    assert torch.equal(cache.k[0, 139999], near.k[0, 0]) and torch.equal(cache.v[0, 139999], near.v[0, 0])
    assert torch.equal(cache.k_scale[0, 139999], near.k_scale[0, 0])


@pytest.mark.parametrize("qlens,klens", [([1, 1], [600, 3000]), ([300, 40], [70, 500]), ([40, 200], [3000, 5000])])
def test_attention_repeats(qlens, klens):
    """The same bits every time, and from a captured graph, replayed after eager
    calls with the table and lengths it then finds."""
    B, cache, q, cu, H = _case(BF16, 128, 64, 4, 1, qlens, klens, seed=19)
    first = _attend(B, cache, q, cu, H)
    for _ in range(3):
        assert torch.equal(_attend(B, cache, q, cu, H), first)
    n = B.attention_cached_workspace_size(cache, cu, H, BF16)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    o = torch.empty_like(q)
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        B.attention_cached(cache, q, o, cu, H, ws, stream=stream)
    table, lens = cache.table.clone(), cache.lens.clone()
    for rep in range(4):
        if rep == 2:   # other requests: the first takes part of the second's pages, the second has none
            cache.table[0, :5] = table[1, :5]
            cache.lens.copy_(_i32([300, 0]))
        o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, _attend(B, cache, q, cu, H)), rep
    assert (o[cu[1]:] == 0).all()
    cache.table.copy_(table)
    cache.lens.copy_(lens)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, first)


def test_tensors_elsewhere_are_refused():
    B, cache, q, cu, H = _case(BF16, 64, 32, 2, 2, [3], [40], seed=3)
    o = torch.empty_like(q)
    for bad in (lambda: B.attention_cached(cache, q.cpu(), o, cu, H), lambda: B.attention_cached(cache, q, o.cpu(), cu, H),
                lambda: B.attention_cached(cache, q, o, cu, H, ws=torch.empty(64, dtype=torch.uint8)),
                lambda: B.cache_store(cache, q, q, torch.zeros(1, 4, dtype=torch.int32))):
        with pytest.raises(ValueError, match="a tensor of"):
            bad()


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("most", [1, 40, 150])
def test_attention_many_requests(dtype, dim, most):
    """As many requests as a call takes, on equal and different lengths, some
    without queries, some without tokens."""
    rng = np.random.default_rng(most)
    qlens = [int(x) for x in rng.integers(0, most + 1, 64)]
    klens = [int(x) for x in rng.choice([0, 1, 18, 64, 64, 65, 200, 517], 64)]
    B, cache, q, cu, H = _case(dtype, dim, 32, 2, 1, qlens, klens, seed=21)
    _check_attention(cache, q, _attend(B, cache, q, cu, H), cu, H, rows=6)


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("qlens,klens", [([9], [100]), ([150], [200]), ([9], [3000]), ([200], [3000])])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_attention_bad_query_rows(dtype, dim, qlens, klens, bad):
    """A query row that is not finite gives a row of NaN, and no other one."""
    B, cache, q, cu, H = _case(dtype, dim, 64, 2, 1, qlens, klens, seed=22)
    log(f"  a value of {bad}")
    q[3, 5] = bad   # of the first head
    o = _attend(B, cache, q, cu, H)
    assert o[3, :dim].isnan().all()
    # the row and head that were spoilt, taken from a call without it
    q[3, 5] = 0
    o[3, :dim] = _attend(B, cache, q, cu, H)[3, :dim]
    _check_attention(cache, q, o, cu, H)


def test_two_calls_at_once():
    """Attention of two batches on two streams, each with its own workspace,
    while a third stream writes another request's pages."""
    B, cache, q, cu, H = _case(BF16, 128, 64, 4, 1, [300, 40], [4000, 700], seed=23)
    spare = int(np.setdiff1d(np.arange(cache.c.n_pages), cache.table.cpu().numpy())[0])   # of neither
    x, _ = _bits(np.random.default_rng(24).standard_normal((64, 4 * 128)), BF16)
    runs = _i32([(spare, 0, 0, 64)])
    few, cu_few = q[:2].contiguous(), [0, 1, 2]
    want = _attend(B, cache, q, cu, H), _attend(B, cache, few, cu_few, H)
    outs = [torch.empty_like(want[0]), torch.empty_like(want[1])]
    ws = [torch.empty(max(B.attention_cached_workspace_size(cache, c, H, BF16), 256), dtype=torch.uint8, device="cuda")
          for c in (cu, cu_few)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for rep in range(20):
        B.attention_cached(cache, q, outs[0], cu, H, ws[0], stream=streams[0])
        B.attention_cached(cache, few, outs[1], cu_few, H, ws[1], stream=streams[1])
        B.cache_store(cache, x, x, runs, stream=streams[2])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_padded_batch_into_the_cache(dtype):
    """Requests' rows at equal distances, the rows behind each one's tokens NaN:
    the same pages as from packed rows."""
    B = require_gpu()
    log(f"case padded batch {dtype}")
    rng = np.random.default_rng(25)
    P, H, d, per, added = 32, 3, 64, 50, [50, 0, 33, 7]
    n = len(added)
    packed, _ = _bits(rng.standard_normal((sum(added), H * d)), dtype)
    padded = torch.full((n * per, H * d), float("nan"), dtype=dtype, device="cuda")
    at = 0
    for r, a in enumerate(added):
        padded[r * per:r * per + a] = packed[at:at + a]
        at += a
    caches = []
    for x, rows_per in ((packed, 0), (padded, per)):
        cache = B.KvCache.empty(8, H, d, P, n, 2)
        runs = torch.empty((B.cache_run_bound(P, n, x.shape[0]), 4), dtype=torch.int32, device="cuda")
        counts = _i32([0] * 4)
        B.cache_tables(cache, None, _i32(added), _i32([7, 1, 4, 2, 0, 3]), runs, counts, x.shape[0], rows_per)
        assert counts.tolist() == [5, 5, 0, sum(added)]
        B.cache_store(cache, x, x, runs)
        caches.append(cache)
    for a, b in zip(*((c.k, c.v, c.k_scale, c.v_scale, c.table, c.lens) for c in caches)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("qlens,klens", [([1] * 12, [9000, 3, 3, 0, 1, 159, 136, 4000, 32, 58, 2, 17]),
                                         ([2, 1, 1, 3], [1, 1, 1, 7000]), ([40, 33, 1, 50], [6000, 3, 0, 900]),
                                         ([129, 1], [64, 8000]), ([1], [20000])])
def test_attention_short_beside_long(dtype, dim, qlens, klens):
    """Shares that hold many short requests, parts of a long one, or only what
    items cost beside their tokens; rows of up to 80 parts."""
    B, cache, q, cu, H = _case(dtype, dim, 64, 3, 1, qlens, klens, seed=26)
    assert B.attention_cached_workspace_size(cache, cu, H, dtype) > 0
    _check_attention(cache, q, _attend(B, cache, q, cu, H), cu, H, rows=12)
