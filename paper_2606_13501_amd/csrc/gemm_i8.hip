// Linear layers on 8-bit integers:
//   out[m][n] = epilogue(sum_k a[m][k] w[n][k] * sa[m] * sw[n] + bias[n]),
// a and w int8 codes, sa a scale for each token, sw one for each output
// channel.  The sum is exact in 32 bits (K is below 2^17, a product at most
// 2^14), so it is the same in whatever order it is added: results depend on no
// tile shape and no split of K.  It is converted to fp32 once, times sa rounded
// to fp32, then one fused multiply-add with sw and bias.
#include <atomic>
#include <type_traits>

#include "common.hpp"
#include "gemm_tiles.hpp"
#include "kernels.hpp"

namespace dit {

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int BK = kRowBytes;   // K step

template <typename T> struct Vec8;   // eight values of an output type
template <> struct Vec8<bf16> { typedef bf16x8 type; };
template <> struct Vec8<float> { typedef float type __attribute__((ext_vector_type(8), aligned(16))); };

// c += w . a^T (or c = w . a^T) for one 16 x 16 block and 64 of K, in place in
// the accumulation registers.  Inline assembly for the reason given at the bf16
// kernel's; the distance to the instructions that read the accumulators is kept
// by hand.
__device__ __forceinline__ void mfma16(i32x4& c, const i32x4& w, const i32x4& a) {
  asm("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(a));
}
__device__ __forceinline__ void mfma16_first(i32x4& c, const i32x4& w, const i32x4& a) {
  asm("v_mfma_i32_16x16x64_i8 %0, %1, %2, 0" : "=a"(c) : "v"(w), "v"(a));
}

// A sum out of the accumulation registers, where it stands: left to the
// compiler, the copies of all 256 would be made at once after the K loop, for
// which the registers do not suffice.
__device__ __forceinline__ int32_t sum_of(const i32x4& c, int e) {
  int32_t v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(c[e]));
  return v;
}

// gelu_tanh(z) = z / (1 + 2^(z (c0 + c1 z^2))), c0 = -2 log2(e) sqrt(2 / pi), c1 =
// 0.044715 c0: two multiplications less than step by step (32,760 x 13,824 x
// 5,120 1.4% faster, in turn).
__device__ __forceinline__ float gelu(float z) {
  constexpr float c0 = -2.302208198f, c1 = -0.1029432397f;
  const float e = __builtin_amdgcn_exp2f(z * fmaf(c1, z * z, c0));   // inf for z << 0: z / inf = 0
  return z * __builtin_amdgcn_rcpf(1.0f + e);
}

// A load from global memory into LDS in two parts, an MFMA between them: the
// address in LDS (m0), then the load itself (16 or 4 bytes a lane).  The vector
// offset passes through the first part so that it is computed there too.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int AT> __device__ __forceinline__ void load_lds_to(uint32_t lds, int& voff) {
  asm volatile("s_add_u32 m0, %1, %2" : "+v"(voff) : "s"(lds), "n"(AT) : "m0", "scc");
}
__device__ __forceinline__ void load_lds_16(const u32x4& desc, int voff, int soff) {
  asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds" :: "v"(voff), "s"(desc), "s"(soff) : "m0");
}
// (A descriptor that the compiler kept in a vector register's lanes comes back
// right before it: five wait states to a load that reads it.)
__device__ __forceinline__ void load_lds_4(const u32x4& desc, int voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "s"(lds), "v"(voff), "s"(desc) : "m0");
}
#pragma clang diagnostic pop

// What an epilogue needs of the call.
template <typename T>
struct Epi {
  const float* sa;
  const float* sw;
  const T* bias;        // or NULL
  T* out; int64_t ldo;
  const T* res; int64_t ldr;
  const float* gate; int64_t gate_stride;
  ReqTable req;
};

// The tiles of a workgroup in tile_seq's order, one after the other without a
// division by a variable per tile: place r of its raster group, whose rows are g
// (below 2^5; r is below 2^27, where r inv >> 32 is r / g).
struct TileWalk {
  int left, r, first_m, g, stride, tiles_m, tiles_n, group_m;
  uint32_t inv;   // ceil(2^32 / g)
  __device__ void group(int m) {
    first_m = m;
    g = min(tiles_m - m, group_m);
    inv = g > 1 ? 0xFFFFFFFFu / (uint32_t)g + 1 : 0;
  }
  __device__ explicit TileWalk(const TileSeq& q)
      : left(q.count), stride(q.stride), tiles_m(q.tiles_m), tiles_n(q.tiles_n), group_m(q.group_m) {
    const int width = group_m * tiles_n;
    r = q.first % width;
    group(q.first / width * group_m);
  }
  __device__ bool next(int& tm, int& tn) {   // false: none is left
    if (left == 0) return false;
    --left;
    while (__builtin_expect(r >= g * tiles_n, 0)) {   // on in a later group
      r -= g * tiles_n;
      group(first_m + g);
    }
    tn = g > 1 ? (int)(((uint64_t)(uint32_t)r * inv) >> 32) : r;
    tm = first_m + r - tn * g;
    r += stride;
    return true;
  }
};

// ------------------------------------------------------------------- tiles
//
// The scheme of the bf16 kernel: a workgroup per compute unit takes a sequence
// of output tiles, operand rows of 128 bytes a step go straight into two LDS
// rings, and a step is two halves of 64 bytes whose fragments are read one half
// ahead.  128 bytes are 128 of K here, and v_mfma_i32_16x16x64_i8 takes the 16
// bytes per lane that v_mfma_f32_16x16x32_bf16 takes, in the same time, for
// twice the products.
//
// Large products run at the board's power limit: 75,600 x 15,360 x 5,120 4,068 us,
// 2.92 PFLOP/s with the matrix cores 78% busy at 1.78 GHz, where a loop of these
// instructions on registers, random operands, reaches 4.1 PFLOP/s at 2.06 GHz; the
// bf16 kernel takes twice as long.  Three steps a turn of the K loop took 3.8% of the
// cycles away and 2.2% of the time, the clock falling meanwhile.  15,209 x 5,120 x
// 13,824, gated, 784 us (its 1,200 tiles take five rounds of 256); 32,760 x 13,824
// x 5,120 with GELU 1,675, 75 of them for the GELU (in turn).
//
// channel_swizzle: the 16 lanes that read the rows 8 a + 4 h + c of W (a, c = 0
// .. 3) at one logical chunk touch 16 distinct bank groups: rows of one parity
// get 8 different chunks.
__device__ __forceinline__ int channel_swizzle(int r) { return (((r >> 3) & 3) << 1) | ((r >> 1) & 1); }

// K need not be whole steps: in the last one, the lanes whose 16 bytes lie
// behind K load from an offset that no descriptor reaches, and get zeros.
constexpr uint32_t kNowhere = 0x80000000u;

template <typename T, int EPI, typename S>
__global__ __launch_bounds__(kThreads, 1) void gemm_i8_nt(
    const int8_t* __restrict__ A, int64_t lda, const int8_t* __restrict__ W, int64_t ldw, Epi<T> ep, int M, int N, int K,
    int tiles_m, int tiles_n, int group_m) {
  typedef typename Vec8<T>::type V8;
  constexpr int MB = S::MB, NB = S::NB, BM = S::BM, BN = S::BN, RX = S::RX, RY = S::RY;
  constexpr int LA = S::LA, LW = S::LW, LX = S::LX, LY = S::LY;
  constexpr bool XA = S::XA;
  __shared__ __attribute__((aligned(1024))) char smem[S::kLds];

  const TileSeq seq = tile_seq(blockIdx.x, gridDim.x, tiles_m, tiles_n, group_m);
  if (seq.count == 0) return;
  TileWalk walk(seq);
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int KT = (K + BK - 1) / BK;
  const int tail_chunks = (K - (KT - 1) * BK) / 16;   // 16-byte chunks of a row in the last step

  // ---- global -> LDS, as in the bf16 kernel: pieces of 8 rows x 128 bytes,
  // lane i of piece q holds row 8 q + i / 8, logical chunk (i % 8) ^ the row's
  // swizzle: row_swizzle for A, whose swizzle is that of the parity of q, and
  // channel_swizzle for W, of q mod 4.  A tile's descriptor ends with the operand's last row, or
  // 2 GiB on: a tile's own rows end before (row strides are at most 2^22).
  static_assert(LA % 2 == 0 && LW % 2 == 0, "the parity of a piece is that of its index in the wave");
  const int a_pc = 8 * (int)lda, w_pc = 8 * (int)ldw;   // bytes of 8 rows
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  // the load cursor: step l_step (l_off bytes on) of its tile, whose coordinates are (l_m, l_n); the lane offsets of that
  // step
  u32x4 ad{}, wd{};
  int l_step = 0, l_off = 0, l_m = 0, l_n = 0;
  int a_at[2], w_at[4];
  auto set_tile = [&]() __attribute__((always_inline)) {
    if (walk.next(l_m, l_n)) {
      ad = make_desc(A + (int64_t)l_m * BM * lda, min((int64_t)0x7FFFFFFF, (int64_t)(M - l_m * BM - 1) * lda + K));
      wd = make_desc(W + (int64_t)l_n * BN * ldw, min((int64_t)0x7FFFFFFF, (int64_t)(N - l_n * BN - 1) * ldw + K));
    } else {   // past the last tile: empty ranges
      ad[2] = 0;
      wd[2] = 0;
    }
  };
  // only a tile's last step differs from the others.  (The lane is hidden from
  // the compiler here and in the epilogue: it would form what depends on it once,
  // before the tiles, and keep that in scratch memory.)
  auto set_step = [&]() __attribute__((always_inline)) {
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int live = l_step == KT - 1 ? tail_chunks : 8;   // chunks of this step; offsets of rows are below 2^30
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c = (ln & 7) ^ row_swizzle(8 * (LA * wave + u) + (ln >> 3));
      a_at[u] = ((LA * wave * 8 + (ln >> 3)) * (int)lda + c * 16) | (c < live ? 0 : (int)kNowhere);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int c = (ln & 7) ^ channel_swizzle(8 * (LW * wave + u) + (ln >> 3));
      w_at[u] = ((LW * wave * 8 + (ln >> 3)) * (int)ldw + c * 16) | (c < live ? 0 : (int)kNowhere);
    }
  };
  auto advance = [&]() __attribute__((always_inline)) {
    l_off += BK;
    if (__builtin_expect(++l_step >= KT - 1, 0)) {
      if (l_step == KT) {
        l_step = l_off = 0;
        set_tile();
      }
      if (tail_chunks < 8) set_step();
    }
  };
  const uint32_t lds_a = lds_base + LA * 1024 * wave, lds_w = lds_base + S::kBaseW + LW * 1024 * wave;
  constexpr int SX = XA ? S::kSlotA : S::kSlotW, SY = XA ? S::kSlotW : S::kSlotA;   // bytes of a slot
  const uint32_t lds_x = XA ? lds_a : lds_w, lds_y = XA ? lds_w : lds_a;

  // ---- fragment reads: logical chunk 4 kk + (lane >> 4) of half kk; of A, row
  // base + 16 b + (lane & 15); of W, the rows that make block pair k of a lane's
  // results eight channels in a row: block 2 k + h takes, as its rows 4 f + e,
  // the channels 32 k + 8 f + 4 h + e.
  static_assert(NB % 2 == 0, "blocks of W come in pairs");
  const int fr = lane & 15, fh = lane >> 4;
  const int wrow = wn * 16 * NB + 8 * (fr >> 2) + (fr & 3);
  int fo_a[2], fo_w[2];             // + 16 * kRowBytes b, + w_block(i)
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    fo_a[kk] = (wm * 16 * MB + fr) * kRowBytes + (((4 * kk + fh) ^ row_swizzle(fr)) << 4);   // the swizzles of all blocks' rows
    fo_w[kk] = S::kBaseW + wrow * kRowBytes + (((4 * kk + fh) ^ channel_swizzle(wrow)) << 4);
  }
  auto w_block = [](int i) { return (32 * (i >> 1) + 4 * (i & 1)) * kRowBytes; };
  struct Frags { i32x4 w[NB], a[MB]; };
  Frags f0, f1;

  // ---- the scales and biases of a tile: the wave's own go into the part of the
  // last step's Y slot that the wave itself refills in the next step, from byte 0
  // (rows), 512 (channels) and 1024 (biases) of it on; behind the last they are zeros.
  auto scales_at = [&](int py) { return (XA ? S::kBaseW : 0) + py + wave * (LY * 1024); };
  const u32x4 sa_d = make_desc(ep.sa, (int64_t)M * 4), sw_d = make_desc(ep.sw, (int64_t)N * 4);
  const u32x4 bias_d = make_desc(ep.bias, ep.bias ? (int64_t)N * (int)sizeof(T) : 0);
  auto load_scales = [&](int m0, int n0, int at) __attribute__((always_inline)) {
    const uint32_t to = lds_base + at;
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int m = 4 * (m0 + wm * 16 * MB + ln), n = 4 * (n0 + wn * 16 * NB + ln), b = (n0 + wn * 16 * NB) * (int)sizeof(T) + 4 * ln;
#pragma unroll
    for (int q = 0; q < (16 * MB + 63) / 64; ++q) load_lds_4(sa_d, m + 256 * q, to + 256 * q);
#pragma unroll
    for (int q = 0; q < (16 * NB + 63) / 64; ++q) load_lds_4(sw_d, n + 256 * q, to + 512 + 256 * q);
#pragma unroll
    for (int q = 0; q < (16 * NB * (int)sizeof(T) + 255) / 256; ++q) load_lds_4(bias_d, b + 256 * q, to + 1024 + 256 * q);
  };
  static_assert(LY >= 4, "the scales fit");
  // acc[2 k + h][j][e] = sum of row m, channel n of the tile, m = 16 MB wm + 16 j + fr, n = 16 NB wn + 32 k + 8 fh + 4 h + e
  i32x4 acc[NB][MB];

  // One half: the MFMAs on f, among them the reads of the next half's fragments
  // into g (from ra and rw on) and the loads of X or Y into the slot at lds,
  // fenced so that the compiler keeps this order; `last` finds the next half's
  // places among the last MFMAs.  A wave issues an instruction
  // every 4 cycles and an MFMA takes 16, so at most three others go between two
  // MFMAs.  The reads are in the order of their use, w0, a0 .., w1 ..; before
  // the barrier (X: false) they end early, so that they have landed there.
  constexpr int NM = MB * NB, NR = MB + NB;
  struct Places { int ra, rw; uint32_t lds; };   // bytes in LDS: the reads of A's and W's fragments, the loads
  auto half = [&](const Frags& f, Frags& g, const Places& at, auto loads_x, auto first, auto&& last) __attribute__((always_inline)) {
    constexpr bool kX = decltype(loads_x)::value, kA = kX == XA;   // kA: the loads are A's
    constexpr int kReadStep = NM >= 64 ? (kX ? 4 : 3) : NM >= 48 && kX ? 3 : 2, kLoads = kX ? LX : LY;
    static_assert((NM - 1) / kReadStep + 1 >= NR && 4 * kLoads <= NM, "all reads and loads are issued");
    int vo[8];
    auto prepare = [&](auto index) __attribute__((always_inline)) {
      constexpr int u = decltype(index)::value;
      vo[u] = kA ? a_at[u & 1] + u * a_pc : w_at[u & 3] + u * w_pc;
      load_lds_to<u * 1024>(at.lds, vo[u]);
    };
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      const int i = m / MB, j = m % MB;
      if (decltype(first)::value) mfma16_first(acc[i][j], f.w[i], f.a[j]);
      else mfma16(acc[i][j], f.w[i], f.a[j]);
      const int r = m / kReadStep;
      if (m % kReadStep == 0 && r < NR) {
        if (r == 0) g.w[0] = *reinterpret_cast<const i32x4*>(smem + at.rw);
        else if (r <= MB) g.a[r - 1] = *reinterpret_cast<const i32x4*>(smem + at.ra + (r - 1) * 16 * kRowBytes);
        else g.w[r - MB] = *reinterpret_cast<const i32x4*>(smem + at.rw + w_block(r - MB));
      }
      const int l = m / 4;
      if (m % 4 == 1 && l < kLoads) {
        switch (l) {   // the index as a constant of the assembly
          case 0: prepare(std::integral_constant<int, 0>{}); break;
          case 1: prepare(std::integral_constant<int, 1>{}); break;
          case 2: prepare(std::integral_constant<int, 2>{}); break;
          case 3: prepare(std::integral_constant<int, 3>{}); break;
          case 4: prepare(std::integral_constant<int, 4>{}); break;
          case 5: prepare(std::integral_constant<int, 5>{}); break;
          case 6: prepare(std::integral_constant<int, 6>{}); break;
          default: prepare(std::integral_constant<int, 7>{}); break;
        }
      }
      if (m % 4 == 3 && l < kLoads) load_lds_16(kA ? ad : wd, vo[l], l_off);
      if (m == NM - 6) last(std::integral_constant<int, 0>{});
      if (m == NM - 4) last(std::integral_constant<int, 1>{});
      if (m == NM - 2) last(std::integral_constant<int, 2>{});
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // the first tile's steps 0 .. R - 1, then the fragments of step 0's first half
  set_tile();
  set_step();
#pragma unroll
  for (int s = 0; s < RX; ++s) {
#pragma unroll
    for (int u = 0; u < LA; ++u) load_lds16(ad, a_at[u & 1] + u * a_pc, l_off, lds_a + s * S::kSlotA + u * 1024);
#pragma unroll
    for (int u = 0; u < LW; ++u) load_lds16(wd, w_at[u & 3] + u * w_pc, l_off, lds_w + s * S::kSlotW + u * 1024);
    advance();
  }
  wait_vmcnt<(RX - 1) * (LX + LY)>();
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NB; ++i) f0.w[i] = *reinterpret_cast<const i32x4*>(smem + fo_w[0] + w_block(i));
#pragma unroll
  for (int j = 0; j < MB; ++j) f0.a[j] = *reinterpret_cast<const i32x4*>(smem + fo_a[0] + j * 16 * kRowBytes);
  // slots of the current step, counted over all tiles, as bytes into the rings,
  // and of the next; tile coordinates as the cursor found them.  A step's first
  // half loads Y(s + R) into the slot of s - 1, its second X(s + R) into that of s.
  int px = 0, py = 0, px1 = RX > 1 ? SX : 0, py1 = SY;
  Places p1{fo_a[1], fo_w[1], lds_y + (RY - 1) * SY}, p2{};
  auto to_second = [&](auto part) __attribute__((always_inline)) {
    constexpr int k = decltype(part)::value;
    if (k == 0) p2.lds = lds_x + px;
    if (k == 1) p2.ra = fo_a[0] + (XA ? px1 : py1);
    if (k == 2) p2.rw = fo_w[0] + (XA ? py1 : px1);
    if (k == 0) asm volatile("" : "+s"(p2.lds));
    if (k == 1) asm volatile("" : "+v"(p2.ra));
    if (k == 2) asm volatile("" : "+v"(p2.rw));
  };
  auto to_first = [&](auto part) __attribute__((always_inline)) {
    constexpr int k = decltype(part)::value;
    if (k == 0) {
      p1.lds = lds_y + py;
      px = px1;
      py = py1;
      p1.ra = fo_a[1] + (XA ? px : py);
    }
    if (k == 1) {
      p1.rw = fo_w[1] + (XA ? py : px);
      px1 = px == (RX - 1) * SX ? 0 : px + SX;
    }
    if (k == 2) py1 = py == (RY - 1) * SY ? 0 : py + SY;
    if (k == 0) asm volatile("" : "+s"(p1.lds));
    if (k == 0) asm volatile("" : "+v"(p1.ra));
    if (k == 1) asm volatile("" : "+v"(p1.rw));
    if (k == 1) asm volatile("" : "+s"(px1));
    if (k == 2) asm volatile("" : "+s"(py1));
  };
  constexpr int kStores = MB * NB / 2;                       // of a wave's epilogue, at least
  constexpr int kPending = (RX - 2) * LX + (RX - 1) * LY;    // loads that may be in flight at a step's barrier
  static_assert(kPending + kStores <= 63, "the counter's range");
  for (int it = 0; it < seq.count; ++it) {
    int tm = l_m, tn = l_n;   // the load cursor is in this tile, or, with few steps a tile, further on
    if (KT <= RX) seq.coords(it, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN;
    half(f0, f1, p1, std::false_type{}, std::true_type{}, to_second);
    // X(s + 1) and Y(s + 1) have to have landed; R - 2 steps of X and R - 1 of Y
    // may still be in flight and, in a tile's first step, the stores of the tile before
    if (it == 0) wait_vmcnt<kPending>();
    else wait_vmcnt<kPending + kStores>();
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
    auto step = [&]() __attribute__((always_inline)) {   // from the middle of a step to that of the next
      half(f1, f0, p2, std::true_type{}, std::false_type{}, to_first);
      advance();
      half(f0, f1, p1, std::false_type{}, std::false_type{}, to_second);
      wait_vmcnt<kPending>();
      __syncthreads();
      __builtin_amdgcn_sched_barrier(0);
    };
    int s = 1;
    for (; s + 2 < KT; s += 3) {   // three steps a turn instead of one: 3.8% of the cycles less
      step();
      step();
      step();
    }
    for (; s < KT; ++s) step();
    const int scales = scales_at(py);   // in the last step's Y slot
    load_scales(m0, n0, scales);
    half(f1, f0, p2, std::true_type{}, std::false_type{}, to_first);
    advance();
    // wait states from the last MFMA to a vector read of its result (the
    // compiler itself would put at most 12), and the scales, which only the last
    // step's X loads follow
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15" ::: "memory");
    wait_vmcnt<LX>();
    __builtin_amdgcn_sched_barrier(0);

    // Epilogue, straight from the accumulators: a lane holds eight channels in a
    // row of each block pair and row, so a wave's store is 16 rows x 64 bytes.
    // Rows behind the last are behind the descriptor's end, channels behind the
    // last at an offset that it does not reach: every wave issues all its stores,
    // which the next tile's first wait counts on.  out may be res: every element
    // is read before it is written, by the same lane.
    constexpr bool kRes = EPI == DIT_EPI_RESIDUAL || EPI == DIT_EPI_GATED_RESIDUAL;
    constexpr int NP = NB / 2, ES = sizeof(T);
    constexpr int kAhead = ES == 2 ? 1 : 0;   // row blocks by which the residual is loaded ahead
    const int mw = m0 + wm * 16 * MB, nw = n0 + wn * 16 * NB;   // the wave's first row and channel
    int el = lane;
    asm volatile("" : "+v"(el));
    const int er = el & 15, eh = el >> 4;
    const char* const sc = smem + scales;
    float wscale[NP][8], bias[NP][8];
    float row_scale[2];   // of this row block and the next
    row_scale[0] = *reinterpret_cast<const float*>(sc + 4 * er);
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const f32x4* const w4 = reinterpret_cast<const f32x4*>(sc + 512 + 4 * (32 * k + 8 * eh));
      const V8 b8 = *reinterpret_cast<const V8*>(sc + 1024 + ES * (32 * k + 8 * eh));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        wscale[k][e] = w4[e / 4][e % 4];
        bias[k][e] = (float)b8[e];
      }
    }
    int out_at[NP], res_at[NP];   // lane offsets inside 16 rows
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const int n = 8 * eh + 32 * k;
      out_at[k] = nw + n < N ? (er * (int)ep.ldo + n) * ES : (int)kNowhere;
      res_at[k] = kRes && nw + n < N ? (er * (int)ep.ldr + n) * ES : (int)kNowhere;
      asm volatile("" : "+v"(out_at[k]), "+v"(res_at[k]));   // formed once
    }
    // the wave's rows 16 j .. 16 j + 15 from its first channel on
    const char* const out0 = (const char*)(ep.out + (int64_t)mw * ep.ldo + nw);
    const char* const res0 = kRes ? (const char*)(ep.res + (int64_t)mw * ep.ldr + nw) : nullptr;
    auto rows_of = [&](const char* p, int64_t ld, int j) {
      return __builtin_amdgcn_make_buffer_rsrc((void*)(p + j * (16 * ES * ld)), 0, max(0, min(16, M - mw - 16 * j)) * (int)ld * ES,
                                               0x00020000);
    };
    f32x4 rv[1 + kAhead][NP][ES / 2];
    auto load_res = [&](int j) __attribute__((always_inline)) {
      if constexpr (kRes) {
        const auto d = rows_of(res0, ep.ldr, j);
#pragma unroll
        for (int k = 0; k < NP; ++k)
#pragma unroll
          for (int q = 0; q < ES / 2; ++q)
            rv[j & kAhead][k][q] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(d, res_at[k] + 16 * q, 0, 0));
      }
    };
    if (kAhead) load_res(0);
    f32x4 gv[NP][2];
    bool g_one = true;   // all rows of the wave belong to one request
    auto load_gate = [&](int r) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        const float* const gp = ep.gate + (int64_t)r * ep.gate_stride + min(nw + 32 * k + 8 * eh, N - 8);
        gv[k][0] = *reinterpret_cast<const f32x4*>(gp);
        gv[k][1] = *reinterpret_cast<const f32x4*>(gp + 4);
      }
    };
    if constexpr (EPI == DIT_EPI_GATED_RESIDUAL) {
      const int r = find_req(ep.req.cu, ep.req.n_req, min(mw, M - 1));
      g_one = r == find_req(ep.req.cu, ep.req.n_req, min(mw + 16 * MB - 1, M - 1));
      load_gate(r);
    }
#pragma unroll
    for (int j = 0; j < MB; ++j) {
      if (j + 1 < MB) row_scale[(j + 1) & 1] = *reinterpret_cast<const float*>(sc + 4 * (16 * (j + 1) + er));
      if (j + kAhead < MB) load_res(j + kAhead);
      if (EPI == DIT_EPI_GATED_RESIDUAL && !g_one) load_gate(find_req(ep.req.cu, ep.req.n_req, min(mw + 16 * j + er, M - 1)));
      const auto d = rows_of(out0, ep.ldo, j);
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        __builtin_amdgcn_sched_barrier(0);   // more of them in flight cost spilled registers
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = fmaf((float)sum_of(acc[2 * k + e / 4][j], e % 4) * row_scale[j & 1], wscale[k][e], bias[k][e]);
        if constexpr (EPI == DIT_EPI_GELU_TANH) {
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = gelu(z[e]);
        } else if constexpr (kRes) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float r = ES == 2 ? (float)__builtin_bit_cast(bf16x8, rv[j & kAhead][k][0])[e] : rv[j & kAhead][k][e / 4 % (ES / 2)][e % 4];
            z[e] = EPI == DIT_EPI_GATED_RESIDUAL ? fmaf(gv[k][e / 4][e % 4], z[e], r) : r + z[e];
          }
        }
        if constexpr (ES == 2) {
          u32x4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{z[2 * e], z[2 * e + 1]}, bf16x2));
          __builtin_amdgcn_raw_buffer_store_b128(o, d, out_at[k], 0, 0);
        } else {
#pragma unroll
          for (int q = 0; q < 2; ++q)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{z[4 * q], z[4 * q + 1], z[4 * q + 2], z[4 * q + 3]}), d,
                                                   out_at[k] + 16 * q, 0, 0);
        }
      }
    }
    // the scales are read before the next step's loads overwrite them, and no store moves behind those loads
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  wait_vmcnt<0>();   // no load may land in LDS after the workgroup has ended
}

// ---------------------------------------------------------------- few rows
//
// Where tiles of 128 x 128 would leave most compute units without work, a
// workgroup computes MB x NB blocks of 16 x 16 only, and its NW waves share K in
// turns of 128 bytes; their sums, whole numbers, meet in LDS.  Each wave has a
// ring of R turns in LDS for itself, filled straight from global memory in whole
// cache lines, so the K loop has no barrier, and the ring runs on into the
// workgroup's next tile while this one's sums are joined.  Bound by the weights'
// bytes, or by the launch: 1 x 30,720 x 5,120 28.2 us with weights from memory (5.6
// TB/s) and 23.6 with the same ones again, partly in the last-level cache; 64 x 384
// x 1,536 in fp32 3.9 us.
template <int MB_, int NB_, int NW_, int R_>
struct FewShape {
  static constexpr int MB = MB_, NB = NB_, NW = NW_, R = R_;
  static constexpr int kLoads = 2 * (MB + NB);                       // 1 KiB loads of a turn
  static constexpr int kSlot = 1024 * kLoads;
  static constexpr int kScales = 768;                                // scales of rows and channels and biases, 256 B each
  static constexpr int kPart = NW * R * kSlot;                       // LDS: rings, partial sums, R + 1 tiles' scales of each wave
  static constexpr int kScalesAt = kPart + NW * MB * NB * 1024;
  static constexpr int kLds = kScalesAt + NW * (R + 1) * kScales;
  static constexpr int kResident = kLds <= 80 * 1024 ? 2 : 1;        // workgroups of a compute unit
  static_assert(MB <= 4 && NB <= 4 && (R - 1) * kLoads <= 63 && kLds <= 160 * 1024, "one load of scales, the counter, LDS");
};

template <typename T, int EPI, typename S>
__global__ __launch_bounds__(64 * S::NW, 1) void gemm_i8_few(
    const int8_t* __restrict__ A, int64_t lda, const int8_t* __restrict__ W, int64_t ldw, Epi<T> ep, int M, int N, int K,
    int tiles_m, int tiles) {
  typedef T V4 __attribute__((ext_vector_type(4)));
  constexpr int MB = S::MB, NB = S::NB, NW = S::NW, R = S::R;
  __shared__ __attribute__((aligned(1024))) char smem[S::kLds];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fh = lane >> 4;
  const int turns = (K + BK - 1) / BK, per_wave = (turns + NW - 1) / NW;   // wave w takes turns w, w + NW, ..
  const int tail_chunks = (K - (turns - 1) * BK) / 16;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int ring = wave * R * S::kSlot, scales = S::kScalesAt + wave * (R + 1) * S::kScales;
  // Tile t: its row tiles are next to each other on one XCD (workgroups go
  // round-robin over the 8), which reads their weights once.
  auto coords = [&](int t, int& m0, int& n0) __attribute__((always_inline)) {
    const int q = t / kXcds, g = q / tiles_m;
    m0 = (q - g * tiles_m) * (16 * MB);
    n0 = (g * kXcds + t % kXcds) * (16 * NB);
  };

  // ---- loads: pieces of 8 rows x 128 bytes, swizzled, as in the tiled kernel
  u32x4 ad{}, wd{};
  const u32x4 sa_d = make_desc(ep.sa, (int64_t)M * 4), sw_d = make_desc(ep.sw, (int64_t)N * 4);
  const u32x4 bias_d = make_desc(ep.bias, ep.bias ? (int64_t)N * (int)sizeof(T) : 0);
  const int a_pc = 8 * (int)lda, w_pc = 8 * (int)ldw;
  int l_tile = blockIdx.x, l_turn = wave, l_left = per_wave, l_slot = 0, l_buf = 0;
  auto set_tile = [&]() __attribute__((always_inline)) {
    if (l_tile < tiles) {
      int m0, n0;
      coords(l_tile, m0, n0);
      ad = make_desc(A + (int64_t)m0 * lda, min((int64_t)0x7FFFFFFF, (int64_t)(M - m0 - 1) * lda + K));
      // (the last tiles of the round-robin order may lie behind the last channel)
      wd = make_desc(W + (int64_t)min(n0, N - 1) * ldw, n0 < N ? min((int64_t)0x7FFFFFFF, (int64_t)(N - n0 - 1) * ldw + K) : 0);
      const uint32_t to = lds_base + scales + l_buf * S::kScales;
      load_lds_4(sa_d, 4 * (m0 + lane), to);
      load_lds_4(sw_d, 4 * (n0 + lane), to + 256);
      load_lds_4(bias_d, n0 * (int)sizeof(T) + 4 * lane, to + 512);
      l_buf = l_buf == R ? 0 : l_buf + 1;
    } else {   // past the last tile
      ad[2] = 0;
      wd[2] = 0;
    }
  };
  auto load = [&]() __attribute__((always_inline)) {   // the cursor's turn into its slot, and the cursor on
    if (l_left == per_wave) set_tile();
    // chunks of this turn: a row's 8, what K leaves of the last one, none behind it
    const int live = l_turn < turns - 1 ? 8 : l_turn == turns - 1 ? tail_chunks : 0;
    const uint32_t to = lds_base + ring + l_slot * S::kSlot;
    int a_at[2], w_at[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c = (lane & 7) ^ row_swizzle(8 * u + (lane >> 3)), none = c < live ? 0 : (int)kNowhere;
      a_at[u] = ((lane >> 3) * (int)lda + c * 16) | none;
      w_at[u] = ((lane >> 3) * (int)ldw + c * 16) | none;
    }
#pragma unroll
    for (int u = 0; u < 2 * MB; ++u) load_lds16(ad, a_at[u & 1] + u * a_pc, l_turn * BK, to + u * 1024);
#pragma unroll
    for (int u = 0; u < 2 * NB; ++u) load_lds16(wd, w_at[u & 1] + u * w_pc, l_turn * BK, to + (2 * MB + u) * 1024);
    l_slot = l_slot == R - 1 ? 0 : l_slot + 1;
    l_turn += NW;
    if (--l_left == 0) {
      l_turn = wave;
      l_left = per_wave;
      l_tile += gridDim.x;
    }
  };
  int fo[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) fo[kk] = fr * kRowBytes + (((4 * kk + fh) ^ row_swizzle(fr)) << 4);

#pragma unroll
  for (int r = 0; r < R; ++r) load();
  int slot = 0, buf = 0;
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    i32x4 acc[NB][MB] = {};
    for (int i = 0; i < per_wave; ++i) {
      wait_vmcnt<(R - 1) * S::kLoads>();   // this turn's loads, and its tile's scales
      i32x4 a[2][MB], w[2][NB];
      const char* const at = smem + ring + slot * S::kSlot;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
        for (int n = 0; n < NB; ++n) w[kk][n] = *reinterpret_cast<const i32x4*>(at + fo[kk] + (MB + n) * 2048);
#pragma unroll
        for (int j = 0; j < MB; ++j) a[kk][j] = *reinterpret_cast<const i32x4*>(at + fo[kk] + j * 2048);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // before the slot is filled again
      load();
      slot = slot == R - 1 ? 0 : slot + 1;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int j = 0; j < MB; ++j) acc[n][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[kk][n], a[kk][j], acc[n][j], 0, 0, 0);
    }
    i32x4* const part = reinterpret_cast<i32x4*>(smem + S::kPart);
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int j = 0; j < MB; ++j) part[(wave * MB * NB + n * MB + j) * 64 + lane] = acc[n][j];
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    int m0, n0;
    coords(tile, m0, n0);
    const char* const sc = smem + scales + buf * S::kScales;
    buf = buf == R ? 0 : buf + 1;
#pragma unroll
    for (int x = 0; x < (MB * NB + NW - 1) / NW; ++x) {
      const int b = wave + NW * x;
      const int ml = 16 * (b % MB) + fr, nl = 16 * (b / MB) + 4 * fh, m = m0 + ml, n = n0 + nl;
      if (b >= MB * NB || m >= M || n >= N) continue;
      i32x4 c = part[b * 64 + lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) c += part[(w * MB * NB + b) * 64 + lane];
      const float sa = *reinterpret_cast<const float*>(sc + 4 * ml);
      const f32x4 sw = *reinterpret_cast<const f32x4*>(sc + 256 + 4 * nl);
      const V4 bias = *reinterpret_cast<const V4*>(sc + 512 + (int)sizeof(T) * nl);
      float z[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = fmaf((float)c[e] * sa, sw[e], (float)bias[e]);
      if (EPI == DIT_EPI_GELU_TANH) {
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = gelu(z[e]);
      } else if (EPI == DIT_EPI_RESIDUAL || EPI == DIT_EPI_GATED_RESIDUAL) {
        const V4 r = *reinterpret_cast<const V4*>(ep.res + (int64_t)m * ep.ldr + n);
        if (EPI == DIT_EPI_GATED_RESIDUAL) {
          const f32x4 g = *reinterpret_cast<const f32x4*>(ep.gate + (int64_t)find_req(ep.req.cu, ep.req.n_req, m) * ep.gate_stride + n);
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] = fmaf(g[e], z[e], (float)r[e]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] = (float)r[e] + z[e];
        }
      }
      V4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (T)z[e];
      *reinterpret_cast<V4*>(ep.out + (int64_t)m * ep.ldo + n) = o;
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // the sums are read before the next tile's are written
  }
  wait_vmcnt<0>();   // no load may land in LDS after the workgroup has ended
}

// -------------------------------------------------------------- the choice

// The tile shapes, by the index of kTiles, and the shapes for few rows, by that of kFew.
typedef Shape<8, 8, 2, false> Tile256x256;
typedef Shape<8, 6, 2, false> Tile256x192;
typedef Shape<4, 8, 2, true> Tile128x256;
typedef Shape<4, 6, 3, false> Tile128x192;
typedef Shape<4, 4, 4, false> Tile128x128;
typedef FewShape<1, 1, 4, 2> Few16x16;
typedef FewShape<2, 2, 4, 3> Few32x32;
typedef FewShape<2, 4, 4, 2> Few32x64;
typedef FewShape<4, 4, 2, 3> Few64x64;

// What a launch takes on 256 compute units, in us.  Of tiles: `launch`, for each
// round of tiles (one per compute unit) `fixed` and per K step `step`, per K step
// and share of the compute units kept busy `busy`, per MB of weights `weights`.
// For few rows: `launch`, for each round (`resident` workgroups per compute unit)
// `fixed` and per turn of a wave `turn`, per MB that all workgroups read together
// `read`, per MB of weights `weights`.
//
// Fitted to 342 products with weights from memory, M = 1 to 32,760, N = 64 to
// 30,720, K = 256 to 14,336, each timed with every shape (as a graph of calls, M
// up to 512): the shape with the least estimate is 1.9% slower than the fastest
// in the mean, 26% at most (17 x 200 x 12,000).  With 9 more shapes for few rows
// (more or fewer waves, 16 x 32, 16 x 64, 32 x 16, 64 x 16, 64 x 32) the best of
// all would be those 1.9% faster.  In us, 128 x 128 and the shapes for few rows:
// 1 x 5,120 x 5,120 21.0 and 8.3 (16 x 16), 64 x 5,120 x 5,120 26.7 and 13.5 (32
// x 64), 128 x 5,120 x 13,824 64.9 and 36.7 (64 x 64), 64 x 384 x 1,536 8.1 and
// 3.3, 1 x 30,720 x 5,120 32.8 and 28.3; but 64 x 30,720 x 5,120 38.1 and 40.8,
// 256 x 15,360 x 5,120 34.0 and 61.0.
struct TileCost { int bm, bn; float launch, fixed, step, busy, weights; };
constexpr TileCost kTiles[5] = {
    {256, 256, 1.11f, 7.02f, 0.938f, 0.339f, 0.060f}, {256, 192, 1.81f, 4.96f, 0.725f, 0.265f, 0.060f},
    {128, 256, 2.27f, 3.12f, 0.566f, 0.200f, 0.143f}, {128, 192, 2.99f, 2.25f, 0.459f, 0.169f, 0.123f},
    {128, 128, 3.32f, 1.42f, 0.339f, 0.165f, 0.083f}};
struct FewCost { int bm, bn, waves, resident; float launch, fixed, turn, read, weights; };
constexpr FewCost kFew[4] = {
    {16, 16, Few16x16::NW, Few16x16::kResident, 2.39f, 0.848f, 0.175f, 0.0180f, 0.095f},
    {32, 32, Few32x32::NW, Few32x32::kResident, 2.76f, 0.783f, 0.299f, 0.0114f, 0.074f},
    {32, 64, Few32x64::NW, Few32x64::kResident, 2.57f, 1.187f, 0.500f, 0.0061f, 0.098f},
    {64, 64, Few64x64::NW, Few64x64::kResident, 2.80f, 2.162f, 0.511f, 0.0043f, 0.047f}};
constexpr int kFewRows = 4096;   // rows up to which the shapes for few rows are launched

std::atomic<int> g_shape{-1};   // forced shape (-1: chosen per call)

// The index of the call's shape: of kTiles, or 5 and that of kFew.
int choose(int64_t M, int N, int K, int cus) {
  const int forced = g_shape.load(std::memory_order_relaxed);
  if (forced >= 0 && (forced < 5 || M <= kFewRows)) return forced;
  auto ceil_div = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  const float kt = (float)ceil_div(K, BK), weights = (float)N * (float)K * 1e-6f;
  int best = 0;
  float least = 0.f;
  for (int t = 0; t < 5; ++t) {
    const TileCost& c = kTiles[t];
    const int64_t tiles = ceil_div(M, c.bm) * ceil_div(N, c.bn);
    const float cost = c.launch + (float)ceil_div(tiles, cus) * (c.fixed + kt * c.step) +
                       kt * (float)tiles / (float)cus * c.busy + weights * c.weights;
    if (t == 0 || cost < least) {
      best = t;
      least = cost;
    }
  }
  for (int t = 0; t < 4 && M <= kFewRows; ++t) {
    const FewCost& c = kFew[t];
    const int64_t tiles = ceil_div(M, c.bm) * ceil_div(ceil_div(N, c.bn), kXcds) * kXcds;
    const float read = (float)tiles * (float)((M < c.bm ? M : c.bm) + c.bn) * (float)K * 1e-6f;
    const float cost = c.launch + (float)ceil_div(tiles, (int64_t)cus * c.resident) * (c.fixed + (float)ceil_div((int64_t)kt, c.waves) * c.turn) +
                       read * c.read + weights * c.weights;
    if (cost < least) {
      best = 5 + t;
      least = cost;
    }
  }
  return best;
}

// Tile rows per raster group: all of them up to 8, so that one XCD reads a tile
// column's weights (589 x 10,240 x 5,120, 5 tile rows, weights from memory: 41.9
// us in groups of 4, 40.1 so; read in all, 131 and 77 MB), and 4 of more.  Of 2, 3,
// 4 and 8, 4 is the fastest or within 1.1% of it for nine products of 16 to 296
// tile rows, in turn (75,600 x 15,360 x 5,120 4,099, 4,064, 4,048 and 4,126 us,
// 75,600 x 5,120 x 13,824 3,598, 3,623, 3,594 and 3,718, 15,209 x 15,360 x 5,120
// 864, 851, 847 and 869).
int raster(int64_t tiles_m) { return tiles_m <= 8 ? (int)tiles_m : 4; }

template <typename T>
Epi<T> epi_of(const LinearI8Args& p) {
  return {p.a_scales, p.w_scales, (const T*)p.bias, (T*)p.out, p.ldo, (const T*)p.res, p.ldr, p.gate, p.gate_stride, p.req};
}

template <typename T, int EPI, typename S>
hipError_t launch_tiles(const LinearI8Args& p, int cus, hipStream_t s) {
  const int64_t tiles_m = (p.M + S::BM - 1) / S::BM, tiles_n = (p.N + S::BN - 1) / S::BN;
  if (tiles_m * tiles_n > 0x7FFFFFF8ll) return hipErrorInvalidValue;
  // one workgroup per compute unit, each running a sequence of tiles
  int grid = (int)((tiles_m * tiles_n + kXcds - 1) / kXcds * kXcds);
  const int resident = cus / kXcds * kXcds;
  if (resident >= kXcds && grid > resident) grid = resident;
  gemm_i8_nt<T, EPI, S><<<grid, kThreads, 0, s>>>(p.a, p.lda, p.w, p.ldw, epi_of<T>(p), (int)p.M, p.N, p.K, (int)tiles_m,
                                                  (int)tiles_n, raster(tiles_m));
  return hipGetLastError();
}

template <typename T, int EPI, typename S>
hipError_t launch_few(const LinearI8Args& p, int cus, hipStream_t s) {
  const int64_t tiles_n = (p.N + 16 * S::NB - 1) / (16 * S::NB), tiles_m = (p.M + 16 * S::MB - 1) / (16 * S::MB);
  const int64_t tiles = (tiles_n + kXcds - 1) / kXcds * kXcds * tiles_m;
  const int64_t resident = (int64_t)cus / kXcds * kXcds * S::kResident;
  const int grid = (int)(resident >= kXcds && tiles > resident ? resident : tiles);
  gemm_i8_few<T, EPI, S><<<grid, 64 * S::NW, 0, s>>>(p.a, p.lda, p.w, p.ldw, epi_of<T>(p), (int)p.M, p.N, p.K, (int)tiles_m,
                                                     (int)tiles);
  return hipGetLastError();
}

template <typename T, int EPI>
hipError_t launch_epi(const LinearI8Args& p, hipStream_t s) {
  const int cus = cu_count();
  switch (choose(p.M, p.N, p.K, cus)) {
    case 0: return launch_tiles<T, EPI, Tile256x256>(p, cus, s);
    case 1: return launch_tiles<T, EPI, Tile256x192>(p, cus, s);
    case 2: return launch_tiles<T, EPI, Tile128x256>(p, cus, s);
    case 3: return launch_tiles<T, EPI, Tile128x192>(p, cus, s);
    case 4: return launch_tiles<T, EPI, Tile128x128>(p, cus, s);
    case 5: return launch_few<T, EPI, Few16x16>(p, cus, s);
    case 6: return launch_few<T, EPI, Few32x32>(p, cus, s);
    case 7: return launch_few<T, EPI, Few32x64>(p, cus, s);
    default: return launch_few<T, EPI, Few64x64>(p, cus, s);
  }
}

template <typename T>
hipError_t launch_typed(const LinearI8Args& p, hipStream_t s) {
  switch (p.epi) {
    case DIT_EPI_NONE: return launch_epi<T, DIT_EPI_NONE>(p, s);
    case DIT_EPI_GELU_TANH: return launch_epi<T, DIT_EPI_GELU_TANH>(p, s);
    case DIT_EPI_RESIDUAL: return launch_epi<T, DIT_EPI_RESIDUAL>(p, s);
    default: return launch_epi<T, DIT_EPI_GATED_RESIDUAL>(p, s);
  }
}

}  // namespace

bool set_linear_i8_tile(int tile_m, int tile_n) {
  int shape = tile_m == 0 && tile_n == 0 ? -1 : -2;
  for (int t = 0; t < 5; ++t)
    if (kTiles[t].bm == tile_m && kTiles[t].bn == tile_n) shape = t;
  for (int t = 0; t < 4; ++t)
    if (kFew[t].bm == tile_m && kFew[t].bn == tile_n) shape = 5 + t;
  if (shape >= -1) g_shape.store(shape, std::memory_order_relaxed);
  return shape >= -1;
}

void linear_i8_plan(int64_t M, int N, int K, int cus, int* tile_m, int* tile_n) {
  const int t = choose(M, N, K, cus);
  *tile_m = t < 5 ? kTiles[t].bm : kFew[t - 5].bm;
  *tile_n = t < 5 ? kTiles[t].bn : kFew[t - 5].bn;
}

hipError_t launch_linear_i8(const LinearI8Args& p, hipStream_t s) {
  if (p.M == 0) return hipSuccess;
  return p.dtype == DIT_BF16 ? launch_typed<bf16>(p, s) : launch_typed<float>(p, s);
}

}  // namespace dit
