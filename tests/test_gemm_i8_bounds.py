"""Extents of the 8-bit GEMM's loads, modelled on the host: the tiled kernel's
loads stay inside their operand for any K (the last step's chunks behind K come
from an offset that no descriptor reaches), offsets hold in 32 bits, and every
chunk of a tile's rows inside K is filled from its own place; the fragment reads
find theirs without bank conflicts, and every output has one lane; the kernel for
few rows reads whole turns inside K and each 16 bytes once."""
import os
import re

import numpy as np
import pytest

SRC = open(os.path.join(os.path.dirname(__file__), "..", "paper_2606_13501_amd", "csrc", "gemm_i8.hip")).read()
BK, WAVES, NOWHERE, FAR = 128, 4, 0x80000000, 0x7FFFFFFF
SHAPES = [(int(a), int(b), int(c), d == "true") for a, b, c, d in re.findall(r"typedef Shape<(\d+), (\d+), (\d+), (true|false)> Tile", SRC)]


def test_constants_are_those_of_the_kernel():
    assert len(SHAPES) == 5
    assert re.search(r"kNowhere = 0x80000000u", SRC) and "constexpr int BK = kRowBytes" in SRC
    assert SRC.count("(int64_t)0x7FFFFFFF") == 2


def row_swizzle(r):
    return (r >> 1) & 7


def channel_swizzle(r):
    return (((r >> 3) & 3) << 1) | ((r >> 1) & 1)


SWIZZLE = {"a": (row_swizzle, 2), "w": (channel_swizzle, 4)}   # and how many lane offsets the kernel keeps


def loads(operand, rows_total, K, ld, blocks, t):
    """The loads of tile t of an operand: (step, lanes that read, byte read, LDS row, physical chunk)."""
    swizzle, kinds = SWIZZLE[operand]
    rows, kt = 32 * blocks, -(-K // BK)
    tail = (K - (kt - 1) * BK) // 16
    m0 = t * rows
    n_rec = min(FAR, (rows_total - m0 - 1) * ld + K)
    lane = np.arange(64)
    for step in {0, max(0, kt - 2), kt - 1}:
        for wave in range(WAVES):
            for u in range(blocks):
                c = (lane & 7) ^ swizzle(8 * (blocks * wave + u % kinds) + (lane >> 3))
                vo = (blocks * wave * 8 + (lane >> 3)) * ld + c * 16
                vo = np.where((step == kt - 1) & (c >= tail), NOWHERE | vo, vo) + u * 8 * ld
                assert vo.max() < 1 << 32
                assert vo[vo < NOWHERE].max(initial=0) < 1 << 30    # int arithmetic in the kernel
                lds = (blocks * wave + u) * 1024 + 16 * lane
                yield step, vo < n_rec, m0 * ld + vo + step * BK, lds // 128, lds % 128 // 16


@pytest.mark.parametrize("operand", ["a", "w"])
@pytest.mark.parametrize("blocks", [8, 6, 4])
@pytest.mark.parametrize("M,K,ld", [
    (1, 16, 16), (1, 128, 128), (300, 144, 160), (257, 112, 112), (512, 272, 4096), (5, 5104, 5120), (255, 131056, 131056),
    (75600, 13824, 13824), (700, 2048, 1 << 22), (256, 48, 1 << 22),
])
def test_loads_stay_inside_and_fill_the_tile(M, K, ld, blocks, operand):
    rows = 32 * blocks
    tiles = -(-M // rows)
    for t in sorted({0, tiles // 2, tiles - 1}):
        filled = set()
        for step, live, at, lds_row, lds_chunk in loads(operand, M, K, ld, blocks, t):
            row, byte = at[live] // ld, at[live] % ld
            assert (row < M).all() and (byte + 16 <= K).all()          # inside the operand and inside K
            chunk = lds_chunk[live] ^ SWIZZLE[operand][0](lds_row[live])
            assert (row == t * rows + lds_row[live]).all() and (byte == step * BK + 16 * chunk).all()
            filled.update(zip([step] * len(row), row.tolist(), byte.tolist()))
        kt = -(-K // BK)
        for step in {0, max(0, kt - 2), kt - 1}:
            want = (min(M, (t + 1) * rows) - t * rows) * (min(K, (step + 1) * BK) - step * BK) // 16
            assert sum(s == step for s, _, _ in filled) == want


@pytest.mark.parametrize("mb,nb,r,xa", SHAPES)
def test_fragment_reads_and_outputs(mb, nb, r, xa):
    """Each read is of the row and chunk that the matrix instruction wants there, 16 lanes at a time in 16 different
    16-byte columns of the banks; the lanes' results are every output of the tile once, eight channels in a row."""
    lane = np.arange(64)
    fr, fh = lane & 15, lane >> 4

    def banks(off):
        for g in range(4):
            assert len(set((off[16 * g:16 * g + 16] % 256 // 16).tolist())) == 16

    for half_wave in range(2):
        for kk in range(2):
            for j in range(mb):
                off = (half_wave * 16 * mb + fr) * 128 + (((4 * kk + fh) ^ row_swizzle(fr)) << 4) + j * 16 * 128
                row = off // 128
                assert (row == half_wave * 16 * mb + 16 * j + fr).all() and row.max() < 32 * mb
                assert (off % 128 // 16 == ((4 * kk + fh) ^ row_swizzle(row))).all()
                banks(off)
            for i in range(nb):
                wrow = half_wave * 16 * nb + 8 * (fr >> 2) + (fr & 3)
                off = wrow * 128 + (((4 * kk + fh) ^ channel_swizzle(wrow)) << 4) + (32 * (i >> 1) + 4 * (i & 1)) * 128
                row = off // 128
                assert (row == half_wave * 16 * nb + 32 * (i // 2) + 8 * (fr // 4) + 4 * (i % 2) + fr % 4).all()
                assert row.max() < 32 * nb
                assert (off % 128 // 16 == ((4 * kk + fh) ^ channel_swizzle(row))).all()
                banks(off)
    # result e of lane (f, g) of block i, j: row fr = f of the A fragment, row 4 g + e of the W fragment
    outs = set()
    for wm in range(2):
        for wn in range(2):
            for i in range(nb):
                for j in range(mb):
                    for g in range(4):
                        for e in range(4):
                            q = 4 * g + e
                            channel = wn * 16 * nb + 32 * (i // 2) + 8 * (q // 4) + 4 * (i % 2) + q % 4
                            assert channel == 16 * nb * wn + 32 * (i >> 1) + 8 * g + 4 * (i & 1) + e   # where the epilogue puts it
                            outs.update((wm * 16 * mb + 16 * j + f, channel) for f in range(16))
    assert len(outs) == 32 * mb * 32 * nb


@pytest.mark.parametrize("mb,nb,r,xa", SHAPES)
@pytest.mark.parametrize("kt", [1, 2, 3, 4, 5, 7])
@pytest.mark.parametrize("bias_loads", [1, 2])
def test_ring_slots_are_free_and_landed(mb, nb, r, xa, kt, bias_loads):
    """A replay of one wave's loads and stores over four tiles of kt steps.  A slot is refilled only after the barrier
    that ends the reads of what it held; a barrier's wait (all but the newest n of the wave's loads and stores) covers
    the next step's operands; the scales go into a free slot, have landed when they are read, and are read before the
    slot is refilled."""
    lx, ly = (mb, nb) if xa else (nb, mb)
    ry, tiles = r + 1, 4
    steps = tiles * kt
    stores, pending = mb * nb // 2, (r - 2) * lx + (r - 1) * ly
    assert pending + stores <= 63
    scale_loads = -(-16 * mb // 64) + -(-16 * nb // 64) + bias_loads
    issued, x, y, free_x, free_y = [], {}, {}, set(), set()

    def issue(what, step):
        ring, slots, free, n = (x, r, free_x, lx) if what == "x" else (y, ry, free_y, ly)
        old = ring.get(step % slots)
        assert old is None or old in free, (what, step, old)
        ring[step % slots] = step
        issued.extend([(what, step)] * n)

    def landed(n, *what):
        done = issued[:len(issued) - n] if n else issued
        for key, count in what:
            assert done.count(key) == count, (key, n)

    for s in range(r):          # the first steps, A's and W's loads in either order
        issue("x", s)
        issue("y", s)
    landed((r - 1) * (lx + ly), (("x", 0), lx), (("y", 0), ly))
    for it in range(tiles):
        for k in range(kt):
            s = it * kt + k
            assert x[s % r] == s and y[s % ry] == s
            if s:
                free_y.add(s - 1)           # read before the last barrier, and the scales in it before the tile ended
            issue("y", s + r)
            landed(pending + (stores if k == 0 and it else 0), (("x", s + 1), lx), (("y", s + 1), ly))
            free_x.add(s)
            if k == kt - 1:                 # the scales: into the slot of Y(s), read by all waves before this barrier
                assert y[s % ry] == s
                issued.extend([("scales", it)] * scale_loads)
            issue("x", s + r)
        landed(lx, (("scales", it), scale_loads))
        assert y[(it * kt + kt - 1) % ry] == it * kt + kt - 1
        issued.extend([("store", it)] * stores)


def test_waits_are_those_of_the_kernel():
    assert "kPending = (RX - 2) * LX + (RX - 1) * LY;" in SRC and "kStores = MB * NB / 2;" in SRC
    assert "if (it == 0) wait_vmcnt<kPending>();" in SRC and "else wait_vmcnt<kPending + kStores>();" in SRC
    assert "wait_vmcnt<LX>();" in SRC


@pytest.mark.parametrize("tiles_m,tiles_n,group_m,nb", [
    (1, 1, 8, 8), (3, 7, 8, 256), (296, 60, 3, 256), (41, 54, 4, 256), (17, 3, 8, 256), (160, 1, 4, 256), (1, 999, 8, 248),
    (9, 131072, 8, 256), (2048, 4, 3, 256), (5, 40, 8, 104)])
def test_a_walk_over_the_tiles_is_tile_seq_s(tiles_m, tiles_n, group_m, nb):
    """The walk without divisions, against the sequence's own coordinates: all tiles once, in the same order."""
    tiles, width, total = tiles_m * tiles_n, group_m * tiles_n, 0
    per_xcd = -(-tiles // 8)
    for b in range(nb):
        lo = b % 8 * per_xcd
        first, stride, hi = lo + b // 8, nb // 8, min(tiles, lo + per_xcd)
        count = -(-(hi - first) // stride) if first < hi else 0
        total += count
        if not count:
            continue
        t = first + stride * np.arange(count)
        group = t // width
        gsize = np.minimum(tiles_m - group * group_m, group_m)
        r = t - group * width
        want_m, want_n = group * group_m + r % gsize, r // gsize
        assert want_m.max() < tiles_m and want_n.max() < tiles_n
        # the walk
        def regroup(m):
            g = min(tiles_m - m, group_m)
            return m, g, (0xFFFFFFFF // g + 1 if g > 1 else 0)
        r, (first_m, g, inv) = first % width, regroup(first // width * group_m)
        for i in range(count if count < 3000 else 300):
            while r >= g * tiles_n:
                r -= g * tiles_n
                first_m, g, inv = regroup(first_m + g)
            tn = r * inv >> 32 if g > 1 else r
            assert (first_m + r - tn * g, tn) == (want_m[i], want_n[i])
            r += stride
    assert total == tiles


FEW = 8


@pytest.mark.parametrize("U", [5, 3, 2])
@pytest.mark.parametrize("K", [16, 64, 112, 128, 144, 1024, 1040, 5120, 5136, 13824, 131056])
def test_few_rows_take_each_byte_once(K, U):
    seen = np.zeros(K // 16, dtype=int)
    whole = K // BK
    fh = np.arange(4)
    for wave in range(FEW):
        t = wave
        while t + FEW * (U - 1) < whole:
            for u in range(U):
                for h in range(2):
                    at = (t + FEW * u) * BK + 64 * h + 16 * fh
                    assert (at + 16 <= K).all()
                    seen[at // 16] += 1
            t += FEW * U
        if t * BK < K:
            for u in range(U):
                if (t + FEW * u) * BK < K:
                    for h in range(2):
                        at = (t + FEW * u) * BK + 64 * h + 16 * fh
                        at = at[at < K]
                        assert (at + 16 <= K).all()
                        seen[at // 16] += 1
            assert (t + FEW * U) * BK >= K          # nothing is left for another round
    assert (seen == 1).all()


def test_few_rows_numbers_are_those_of_the_kernel():
    assert f"kFewWaves = {FEW};" in SRC and "U = MB * NB <= 2 ? 5 : MB * NB <= 4 ? 3 : 2" in SRC
