"""CPU oracle (float64, NumPy) of the paged 8-bit key/value cache -- TEST
INFRASTRUCTURE ONLY.  Only the tests may import it; the library's kernels share
no code with it.

What it computes.  ``tables``: pages for the requests' new tokens and the slot
map, one request after another.  ``store``: the codes and scale bytes of a
page after tokens were added, token by token.  ``gather``: a request's cached
tokens as numbers.  ``attention``: the softmax average over them.

A code is a float8 e4m3 number: sign, 4 exponent bits (bias 7), 3 fraction
bits, no infinities, 0x7F / 0xFF NaN, largest 448.  Pins
(tests/test_oracle_cache.py): the code table against its bit fields, every code
and every middle between two codes under rounding, store followed by gather
against a direct rounding of the input, and the placement of tokens by hand.
"""
import numpy as np

SCALE_MIN, TOP = 27, 448.0


def _code_values():
    v = np.empty(256)
    for b in range(256):
        e, f = (b >> 3) & 15, b & 7
        x = np.nan if (e == 15 and f == 7) else (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        v[b] = -x if b & 128 else x
    return v


VALUES = _code_values()


def codes(x):
    """The nearest code, ties to the even one; |x| <= 448 or not finite (NaN)."""
    x = np.asarray(x, np.float64)
    pos = VALUES[:127]                                  # 0 .. 448, increasing
    a = np.where(np.isfinite(x), np.abs(x), 0)
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    lo = hi - 1
    up, down = pos[hi] - a, a - pos[lo]
    c = np.where(up < down, hi, np.where(down < up, lo, np.where(lo % 2 == 0, lo, hi)))
    c = np.where(np.signbit(x), c + 128, c)
    return np.where(np.isfinite(x), c, 127).astype(np.uint8)


def scale_byte(x):
    """Smallest s >= SCALE_MIN with |x| <= 448 * 2^(s - 127) for every finite x."""
    x = np.abs(np.asarray(x, np.float64))
    top = x[np.isfinite(x)].max(initial=0.0)
    s = SCALE_MIN
    while top > TOP * 2.0 ** (s - 127):
        s += 1
    return s


def tables(page_tokens, table, lens_before, added, free_pages, n_rows, rows_per_req=0):
    """Returns (table, lens, runs, counts); the table is a changed copy."""
    P, table = page_tokens, np.array(table)
    cap = table.shape[1] * P
    out = list(lens_before)
    runs, at, short, taken, refused, placed, row = [], 0, False, 0, 0, 0, 0
    for r, (b, a) in enumerate(zip(lens_before, added)):
        b, a = int(b), int(a)
        row0 = r * rows_per_req if rows_per_req else row
        row += max(a, 0)
        fits = a >= 0 and b >= 0 and b + a <= cap and (a <= rows_per_req if rows_per_req else row0 + a <= n_rows)
        if fits:
            have, want = -(-b // P), -(-(b + a) // P) - -(-b // P)
            if want and (short or at + want > len(free_pages)):
                short, fits = True, False
        if not fits:
            refused += 1
            out[r] = min(max(b, 0), cap)
            continue
        for i in range(want):
            table[r, have + i] = free_pages[at + i]
        at, taken, placed, out[r] = at + want, taken + want, placed + a, b + a
        t = b
        while t < b + a:
            n = min((t // P + 1) * P, b + a) - t
            runs.append((int(table[r, t // P]), row0 + t - b, t % P, n))
            t += n
    return table, out, runs, [taken, len(runs), refused, placed]


def k_place(token, channel):
    """Index of a page's key element in [groups, head_dim / 16, 32, 16]."""
    return token // 32, channel // 16, token % 32, channel % 16


def v_place(token, channel):
    """Index of a page's value element in [groups, 2, head_dim, 16]."""
    u = token % 32
    return token // 32, (u // 4) % 2, channel, 4 * (u // 8) + u % 4


def _places(P, head_dim, place):
    t, c = np.meshgrid(np.arange(P), np.arange(head_dim), indexing="ij")
    return place(t, c)


def store(page, scale, new, offset, place):
    """One page and head: ``page`` codes in the cache's layout, ``scale`` its
    byte, ``new`` [count, head_dim] the tokens for places offset ...  Returns
    (codes, scale byte)."""
    groups, head_dim = page.shape[0], new.shape[1]
    idx = _places(32 * groups, head_dim, place)
    tok = page[idx]                                      # [token, channel]
    s = scale_byte(new)
    if offset:
        old = min(max(int(scale), SCALE_MIN), 247)
        s = max(s, old)
        if s > old:
            tok[:offset] = codes(VALUES[tok[:offset]] * 2.0 ** (old - s))
    tok[offset:offset + len(new)] = codes(np.asarray(new, np.float64) * 2.0 ** (127 - s))
    out = page.copy()
    out[idx] = tok
    return out, s


def gather(k, v, k_scale, v_scale, table_row, length, head):
    """A request's cached tokens of one head, as numbers: (K, V, there) of
    ``length`` tokens; ``there`` is False for tokens on pages outside the pool."""
    n_pages, groups = k.shape[0], k.shape[2]
    P, d = 32 * groups, 16 * k.shape[3]
    K, V, there = np.zeros((length, d)), np.zeros((length, d)), np.zeros(length, bool)
    ki, vi = _places(P, d, k_place), _places(P, d, v_place)
    for i in range(-(-length // P)):
        p, n = int(table_row[i]), min(P, length - i * P)
        if not 0 <= p < n_pages:
            continue
        rows = slice(i * P, i * P + n)
        K[rows] = VALUES[k[p, head][ki]][:n] * 2.0 ** (int(k_scale[p, head]) - 127)
        V[rows] = VALUES[v[p, head][vi]][:n] * 2.0 ** (int(v_scale[p, head]) - 127)
        there[rows] = True
    return K, V, there


def attention(q, K, V, there, scale):
    """[n, d] queries over the tokens that are there; rows of zeros without any.
    Also returns the probabilities."""
    K, V = K[there], V[there]
    if len(K) == 0:
        return np.zeros((len(q), V.shape[1])), np.zeros((len(q), 0))
    s = q @ K.T * scale
    p = np.exp(s - s.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    return p @ V, p
