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
    assert SRC.count("(int64_t)0x7FFFFFFF") == 4


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


FEW = [tuple(int(x) for x in m) for m in re.findall(r"typedef FewShape<(\d+), (\d+), (\d+), (\d+)> Few", SRC)]


def test_few_shapes():
    assert len(FEW) == 4
    for mb, nb, nw, r in FEW:
        loads = 2 * (mb + nb)
        lds = nw * r * loads * 1024 + nw * mb * nb * 1024 + nw * (r + 1) * 768
        assert lds <= 160 * 1024 and (r - 1) * loads <= 63 and mb <= 4 and nb <= 4
        # scales: 64 floats for at most 64 rows and channels, 64 floats or 128 bf16 of biases
        assert 16 * max(mb, nb) * 4 <= 256


@pytest.mark.parametrize("operand", ["a", "w"])
@pytest.mark.parametrize("blocks", [1, 2, 4])
@pytest.mark.parametrize("nw", [2, 4])
@pytest.mark.parametrize("M,K,ld", [(1, 16, 16), (1, 128, 128), (40, 144, 160), (64, 112, 112), (65, 272, 4096), (5, 5104, 5120),
                                    (63, 131056, 131056), (100, 2048, 1 << 22), (64, 48, 1 << 22)])
def test_few_rows_loads_stay_inside_and_take_each_byte_once(M, K, ld, nw, blocks, operand):
    rows, turns = 16 * blocks, -(-K // BK)
    per_wave, tail = -(-turns // nw), (K - (turns - 1) * BK) // 16
    lane = np.arange(64)
    for m0 in range(0, M, rows):
        n_rec = min(FAR, (M - m0 - 1) * ld + K)
        seen = np.zeros((min(rows, M - m0), K // 16), dtype=int)
        for wave in range(nw):
            for t in range(wave, wave + nw * per_wave, nw):
                live = 8 if t < turns - 1 else tail if t == turns - 1 else 0
                if K > 20000 and 1 < t < turns - 2:      # the middle is like its neighbours
                    seen[:, t * 8:t * 8 + 8] += 1
                    continue
                for u in range(2 * blocks):
                    c = (lane & 7) ^ row_swizzle(8 * (u & 1) + (lane >> 3))
                    vo = (((lane >> 3) * ld + c * 16) | np.where(c < live, 0, NOWHERE)) + u * 8 * ld
                    assert vo.max() < 1 << 32 and vo[vo < NOWHERE].max(initial=0) < 1 << 30
                    ok = vo < n_rec
                    at = vo[ok] + t * BK
                    row, byte = at // ld, at % ld
                    assert (row < M - m0).all() and (byte + 16 <= K).all()
                    lds = u * 1024 + 16 * lane[ok]           # the fragment reads' place for it
                    assert (lds // 128 == row).all()
                    assert (lds % 128 // 16 ^ row_swizzle(lds // 128) == byte % 128 // 16).all()
                    np.add.at(seen, (row, byte // 16), 1)
        assert (seen == 1).all()


@pytest.mark.parametrize("mb,nb,nw,r", FEW)
@pytest.mark.parametrize("per_wave", [1, 2, 3, 5, 11])
def test_few_rows_ring_and_scales(mb, nb, nw, r, per_wave):
    """One wave's loads over several tiles: each turn's and its tile's scales have landed at its wait, a slot is refilled
    after its reads, a tile's scales stay until its results are written."""
    loads, tiles = 2 * (mb + nb), 9
    issued, slots, bufs = [], {}, {}
    cursor = {"tile": 0, "left": per_wave, "slot": 0, "buf": 0, "turn": 0}

    def load(free_turn, done_tile):
        if cursor["left"] == per_wave and cursor["tile"] < tiles:
            old = bufs.get(cursor["buf"])
            assert old is None or old < done_tile      # its results are written
            bufs[cursor["buf"]] = cursor["tile"]
            issued.extend([("scales", cursor["tile"])] * 3)
            cursor["buf"] = 0 if cursor["buf"] == r else cursor["buf"] + 1
        old = slots.get(cursor["slot"])
        assert old is None or old <= free_turn
        slots[cursor["slot"]] = cursor["turn"]
        issued.extend([("turn", cursor["turn"])] * loads)
        cursor["turn"] += 1
        cursor["slot"] = 0 if cursor["slot"] == r - 1 else cursor["slot"] + 1
        cursor["left"] -= 1
        if cursor["left"] == 0:
            cursor["left"], cursor["tile"] = per_wave, cursor["tile"] + 1

    for _ in range(r):
        load(-1, 0)
    slot = buf = turn = 0
    for tile in range(tiles):
        for _ in range(per_wave):
            done = issued[:len(issued) - (r - 1) * loads]
            assert done.count(("turn", turn)) == loads and done.count(("scales", tile)) == 3
            assert slots[slot] == turn
            load(turn, tile)
            slot = 0 if slot == r - 1 else slot + 1
            turn += 1
        assert bufs[buf] == tile
        buf = 0 if buf == r else buf + 1
        issued.extend([("store", tile)] * (mb * nb // nw))


@pytest.mark.parametrize("tiles_m,tiles_n", [(1, 1), (1, 8), (2, 9), (3, 320), (64, 17), (5, 63)])
def test_few_rows_tiles_cover_the_output(tiles_m, tiles_n):
    groups = -(-tiles_n // 8) * 8
    seen = set()
    for t in range(groups * tiles_m):
        g = t // 8 // tiles_m
        m, n = t // 8 - g * tiles_m, g * 8 + t % 8
        assert n < groups and (m, n) not in seen
        seen.add((m, n))
    assert {(m, n) for m, n in seen if n < tiles_n} == {(m, n) for m in range(tiles_m) for n in range(tiles_n)}
