"""Extents of the 8-bit GEMM's loads, modelled on the host: the tiled kernel's
loads stay inside their operand for any K (the last step's chunks behind K come
from an offset that no descriptor reaches), offsets hold in 32 bits, and every
chunk of a tile's rows inside K is filled from its own place; the kernel for few
rows reads whole turns inside K and each 16 bytes once; the output windows have
a place for every chunk and every row and column one lane."""
import os
import re

import numpy as np
import pytest

SRC = open(os.path.join(os.path.dirname(__file__), "..", "paper_2606_13501_amd", "csrc", "gemm_i8.hip")).read()
BK, WAVES, NOWHERE, FAR = 128, 4, 0x80000000, 0x7FFFFFFF
SHAPES = [tuple(int(x) for x in m) for m in re.findall(r"typedef Shape<(\d+), (\d+), (\d+), (?:true|false)> Tile", SRC)]


def test_constants_are_those_of_the_kernel():
    assert len(SHAPES) == 5
    assert re.search(r"kNowhere = 0x80000000u", SRC) and "constexpr int BK = kRowBytes" in SRC
    assert SRC.count("(int64_t)0x7FFFFFFF") == 2


def loads(rows_total, K, ld, blocks, t):
    """The loads of tile t of an operand: (first byte read or None, LDS row, physical chunk, step) per lane."""
    rows, kt = 32 * blocks, -(-K // BK)
    tail = (K - (kt - 1) * BK) // 16
    m0 = t * rows
    n_rec = min(FAR, (rows_total - m0 - 1) * ld + K)
    lane = np.arange(64)
    for step in {0, max(0, kt - 2), kt - 1}:
        for wave in range(WAVES):
            for u in range(blocks):
                c = (lane & 7) ^ (4 * (u & 1) + (lane >> 4))
                vo = (blocks * wave * 8 + (lane >> 3)) * ld + c * 16
                vo = np.where((step == kt - 1) & (c >= tail), NOWHERE | vo, vo) + u * 8 * ld
                assert vo.max() < 1 << 32
                assert vo[vo < NOWHERE].max(initial=0) < 1 << 30    # int arithmetic in the kernel
                live = vo < n_rec
                at = m0 * ld + vo + step * BK
                lds = (blocks * wave + u) * 1024 + 16 * lane
                yield step, live, at, lds // 128, lds % 128 // 16, vo < NOWHERE


@pytest.mark.parametrize("blocks", [8, 6, 4])
@pytest.mark.parametrize("M,K,ld", [
    (1, 16, 16), (1, 128, 128), (300, 144, 160), (257, 112, 112), (512, 272, 4096), (5, 5104, 5120), (255, 131056, 131056),
    (75600, 13824, 13824), (700, 2048, 1 << 22), (256, 48, 1 << 22),
])
def test_loads_stay_inside_and_fill_the_tile(M, K, ld, blocks):
    rows = 32 * blocks
    tiles = -(-M // rows)
    for t in sorted({0, tiles // 2, tiles - 1}):
        filled = set()
        for step, live, at, lds_row, lds_chunk, asked in loads(M, K, ld, blocks, t):
            row, byte = at[live] // ld, at[live] % ld
            assert (row < M).all() and (byte + 16 <= K).all()          # inside the operand and inside K
            chunk = lds_chunk[live] ^ ((lds_row[live] >> 1) & 7)       # the fragment reads' swizzle
            assert (row == t * rows + lds_row[live]).all() and (byte == step * BK + 16 * chunk).all()
            filled.update(zip([step] * len(row), row.tolist(), byte.tolist()))
        kt = -(-K // BK)
        for step in {0, max(0, kt - 2), kt - 1}:
            want = (min(M, (t + 1) * rows) - t * rows) * (min(K, (step + 1) * BK) - step * BK) // 16
            assert sum(s == step for s, _, _ in filled) == want


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


@pytest.mark.parametrize("mb,nb,r", SHAPES)
def test_output_windows(mb, nb, r):
    """Every value of a wave's block has one place in its windows, written once and read once."""
    xa = (mb, nb) == (4, 8)
    ly = nb if xa else mb
    cw = 64 if nb % 4 == 0 and ly >= 8 else 32
    lane = np.arange(64)
    wr, wh = lane & 15, lane >> 4

    def at(r_, c):
        if cw == 64:
            return r_ * 256 + ((((c >> 1) | ((c & 1) << 3)) ^ (((r_ & 1) << 3) | ((r_ >> 1) & 7))) << 4)
        return r_ * 128 + ((((c >> 1) | ((c & 1) << 2)) ^ ((((r_ >> 1) & 1) << 2) | ((r_ >> 2) & 3))) << 4)

    window = {}
    for ii in range(cw // 16):
        for jj in range(2):
            for l in range(64):
                a = int(at(16 * jj + wr[l], 4 * ii + wh[l]))
                assert a not in window and a + 16 <= ly * 1024
                window[a] = (16 * jj + wr[l], 16 * ii + 4 * wh[l])     # row, first column
    lpr, rpp = cw // 8, 64 // (cw // 8)
    for p in range(32 // rpp):
        for l in range(64):
            row, ec = rpp * p + l // lpr, l % lpr
            for half in range(2):
                assert window.pop(int(at(np.int64(row), np.int64(2 * ec + half)))) == (row, 8 * ec + 4 * half)
    assert not window
