"""Pins of the cache oracle (``oracle.cache``)."""
import numpy as np

from oracle import cache as C


def test_code_table():
    assert C.VALUES[0] == 0 and C.VALUES[1] == 2.0 ** -9 and C.VALUES[7] == 7 * 2.0 ** -9 and C.VALUES[8] == 2.0 ** -6
    assert C.VALUES[0x38] == 1 and C.VALUES[0x7E] == 448 and np.isnan(C.VALUES[0x7F]) and C.VALUES[0xB8] == -1
    assert (np.diff(C.VALUES[:127]) > 0).all()


def test_rounding():
    pos = C.VALUES[:127]
    assert np.array_equal(C.codes(pos), np.arange(127))
    assert np.array_equal(C.codes(-pos[1:]), np.arange(1, 127) + 128)
    mid = (pos[1:] + pos[:-1]) / 2
    assert (C.codes(mid) % 2 == 0).all(), "ties go to the even code"
    assert np.array_equal(C.codes(np.nextafter(mid, 0)), np.arange(126))
    assert np.array_equal(C.codes(np.nextafter(mid, 1e9)), np.arange(1, 127))
    assert (C.codes([np.inf, -np.inf, np.nan]) == 127).all()


def test_scale_byte():
    assert C.scale_byte([448.0]) == 127 and C.scale_byte([-448.5]) == 128 and C.scale_byte([224.0]) == 126
    assert C.scale_byte([0.0]) == C.scale_byte([]) == C.scale_byte([1e-40]) == 27
    assert C.scale_byte([np.inf, np.nan, 1.0]) == 127 - 8
    assert C.scale_byte([3.38e38]) == 247


def test_places_cover_the_page():
    for place, shape in ((C.k_place, (2, 4, 32, 16)), (C.v_place, (2, 2, 64, 16))):
        seen = np.zeros(shape, int)
        for t in range(64):
            for c in range(64):
                seen[place(t, c)] += 1
        assert (seen == 1).all()
    assert C.k_place(37, 50) == (1, 3, 5, 2)
    assert C.v_place(32 + 8 * 3 + 4 + 2, 50) == (1, 1, 50, 14)


def test_store_and_gather():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((45, 64)) * 3
    page = np.full((2, 4, 32, 16), 0x7F, np.uint8)
    got, s = C.store(page, 0, x, 0, C.k_place)
    step = 2.0 ** (s - 127)
    k = got[None, None]
    v, _ = C.store(np.zeros((2, 2, 64, 16), np.uint8), 0, x, 0, C.v_place)
    K, V, there = C.gather(k, v[None, None], np.array([[s]]), np.array([[s]]), [0], 45, 0)
    want = C.VALUES[C.codes(x / step)] * step
    assert np.array_equal(K, want) and np.array_equal(V, want) and there.all()
    assert (np.abs(K - x) <= np.maximum(np.abs(x) * 2.0 ** -4, step * 2.0 ** -10)).all()
    assert (got[1, :, 13:] == 0x7F).all(), "places behind the tokens keep their bytes"
    # continued: a larger value raises the scale, the earlier codes follow
    more, s2 = C.store(got, s, 100 * x[:3], 45, C.k_place)
    assert s2 > s
    K2, _, _ = C.gather(more[None, None], v[None, None], np.array([[s2]]), np.array([[s]]), [0], 48, 0)
    small = np.abs(K) < 2.0 ** (s2 - 127 - 6)
    assert np.array_equal(K2[:45][~small], K[~small])
    # continued with smaller values: the scale stays
    assert C.store(got, s, x[:3] / 100, 45, C.k_place)[1] == s


def test_tables_by_hand():
    t = np.full((3, 3), -1)
    t[0, 0] = 9
    tab, lens, runs, counts = C.tables(32, t, [20, 0, 0], [30, 0, 65], [4, 5, 6, 7], 95)
    assert lens == [50, 0, 65] and counts == [4, 5, 0, 95]
    assert runs == [(9, 0, 20, 12), (4, 12, 0, 18), (5, 30, 0, 32), (6, 62, 0, 32), (7, 94, 0, 1)]
    assert tab.tolist() == [[9, 4, -1], [-1, -1, -1], [5, 6, 7]]
    # too few pages: the second request is refused, the third too although one page would do; the first needs none
    tab, lens, runs, counts = C.tables(32, t, [20, 0, 0], [5, 65, 1], [4, 5], 71)
    assert lens == [25, 0, 0] and counts == [0, 1, 2, 5] and runs == [(9, 0, 20, 5)]
    # a table row that is too short does not stop the others
    assert C.tables(32, t, [0, 0, 0], [97, 1, 1], [4, 5], 99)[3] == [2, 2, 1, 2]


def test_attention():
    rng = np.random.default_rng(2)
    q, K, V = rng.standard_normal((3, 64)), rng.standard_normal((5, 64)), rng.standard_normal((5, 64))
    o, p = C.attention(q, K, V, np.array([True, False, True, False, False]), 0.0)
    assert np.allclose(o, (V[0] + V[2]) / 2) and np.allclose(p, 0.5)
    assert (C.attention(q, K, V, np.zeros(5, bool), 1.0)[0] == 0).all()
    o, _ = C.attention(q, K, V, np.ones(5, bool), 1e4)
    assert np.allclose(o, V[(q @ K.T).argmax(1)])
