// What the tiled GEMM kernels share, whatever their operands' type: the order
// in which workgroups take output tiles, the loads from global memory straight
// into LDS and the tile shapes.  An operand tile's row is 128 bytes of K per step.
#pragma once

#include "common.hpp"

namespace dit {

namespace {

constexpr int kWaves = 4;                           // 2 x 2 waves
constexpr int kThreads = 64 * kWaves;
constexpr int kRowBytes = 128;                      // one full cache line per tile row and K step
constexpr int kXcds = 8;                            // gfx950: 8 XCDs, workgroups dispatched round-robin

// Tile sequence of a workgroup.  Each XCD owns a contiguous range of logical
// tiles (the dispatcher places workgroup b on XCD b mod 8); the workgroups of
// one XCD take its tiles round-robin, so at any time they work on adjacent
// tiles.  Logical tiles are rastered in groups of group_m tile rows, so the
// tiles resident on one XCD share A and W panels in its L2.
struct TileSeq {
  int first, stride, count;   // logical tiles first + stride * it, it < count
  int tiles_m, tiles_n, group_m;
  __device__ void coords(int it, int& tm, int& tn) const {
    const int t = first + stride * it;
    const int width = group_m * tiles_n;
    const int group = t / width;
    const int first_m = group * group_m;
    const int gsize = min(tiles_m - first_m, group_m);
    const int r = t - group * width;
    tm = first_m + r % gsize;
    tn = r / gsize;
  }
};

__device__ __forceinline__ TileSeq tile_seq(int b, int nb, int tiles_m, int tiles_n, int group_m) {
  const int tiles = tiles_m * tiles_n;
  const int per_xcd = (tiles + kXcds - 1) / kXcds;
  const int x = b % kXcds, slot = b / kXcds, wgs = nb / kXcds;
  const int lo = x * per_xcd, hi = min(tiles, lo + per_xcd);
  TileSeq q;
  q.first = lo + slot;
  q.stride = wgs;
  q.count = q.first < hi ? (hi - q.first + wgs - 1) / wgs : 0;
  q.tiles_m = tiles_m;
  q.tiles_n = tiles_n;
  q.group_m = group_m;
  return q;
}

// 16-byte chunk swizzle of a 128-byte LDS row: the 16 lanes that read 16
// consecutive rows at one logical chunk touch, with rows 2t and 2t + 1 in
// different halves of a 256-byte bank window and the physical chunk c ^ t
// different for the 8 values of t, 16 distinct bank groups.
__device__ __forceinline__ int row_swizzle(int r) { return (r >> 1) & 7; }

// Raw buffer descriptor over `bytes` bytes from `base`.  The hardware's range
// check covers the lane offset only (not the scalar offset), so a load
// returns zeros where its lane offset is past the end; the loads below carry
// every row offset in the lane offset.
__device__ __forceinline__ u32x4 make_desc(const void* base, int64_t bytes) {
  const uint32_t n = bytes > 0xFFFFFFFFll ? 0xFFFFFFFFu : (uint32_t)(bytes < 0 ? 0 : bytes);
  const uint64_t p = (uint64_t)base;
  return u32x4{(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, n, 0x00020000u};
}

// 16 bytes per lane from global memory straight into LDS: lane i writes LDS
// bytes lds + 16 i .. +15.  Inline assembly, so the compiler does not make
// later LDS reads wait for it; completion is waited for by hand.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds16(const u32x4& desc, int voff, int soff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :: "s"(lds), "v"(voff), "s"(desc), "s"(soff) : "m0");
}
#pragma clang diagnostic pop
template <int N> __device__ __forceinline__ void wait_vmcnt() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

// A tile shape: each of the 2 x 2 waves owns MB x NB blocks of 16 x 16, the X
// operand (A if XA, else W) has R ring slots and the other one R + 1.
template <int MB_, int NB_, int R_, bool XA_>
struct Shape {
  static constexpr int MB = MB_, NB = NB_, RX = R_, RY = R_ + 1;
  static constexpr bool XA = XA_;
  static constexpr int BM = 32 * MB, BN = 32 * NB;
  static constexpr int kSlotA = BM * kRowBytes, kSlotW = BN * kRowBytes;
  static constexpr int RA = XA ? RX : RY, RW = XA ? RY : RX;
  static constexpr int kBaseW = RA * kSlotA;                 // LDS: the ring of A, then the ring of W
  static constexpr int kLds = kBaseW + RW * kSlotW;
  static constexpr int LA = MB, LW = NB;                     // 1 KiB loads per wave and step
  static constexpr int LX = XA ? LA : LW, LY = XA ? LW : LA;
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
};

}  // namespace

}  // namespace dit
