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

// c += w . a^T for one 16 x 16 block and 64 of K, in place in the accumulation
// registers.  Inline assembly for the reason given at the bf16 kernel's; the
// distances to the instructions that write and read the accumulators are kept
// by hand.
__device__ __forceinline__ void mfma16(i32x4& c, const i32x4& w, const i32x4& a) {
  asm("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(a));
}

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

// ------------------------------------------------------------------- tiles
//
// The scheme of the bf16 kernel: a workgroup per compute unit takes a sequence
// of output tiles, operand rows of 128 bytes a step go straight into two LDS
// rings, and a step is two halves of 64 bytes whose fragments are read one half
// ahead.  128 bytes are 128 of K here, and v_mfma_i32_16x16x64_i8 takes the 16
// bytes per lane that v_mfma_f32_16x16x32_bf16 takes, in the same time, for
// twice the products.
//
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
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int KT = (K + BK - 1) / BK;
  const int tail_chunks = (K - (KT - 1) * BK) / 16;   // 16-byte chunks of a row in the last step

  // ---- global -> LDS, as in the bf16 kernel: pieces of 8 rows x 128 bytes,
  // lane i of piece q holds row 8 q + i / 8, logical chunk (i % 8) ^
  // row_swizzle(row).  A tile's descriptor ends with the operand's last row, or
  // 2 GiB on: a tile's own rows end before (row strides are at most 2^22).
  static_assert(LA % 2 == 0 && LW % 2 == 0, "the parity of a piece is that of its index in the wave");
  int a_vo[2], w_vo[2], behind[2];   // behind: kNowhere if the lane's chunk of the last step is behind K
#pragma unroll
  for (int par = 0; par < 2; ++par) {
    const int c = (lane & 7) ^ (4 * par + (lane >> 4));
    a_vo[par] = (LA * wave * 8 + (lane >> 3)) * (int)lda + c * 16;
    w_vo[par] = (LW * wave * 8 + (lane >> 3)) * (int)ldw + c * 16;
    behind[par] = c < tail_chunks ? 0 : (int)kNowhere;
  }
  const int a_pc = 8 * (int)lda, w_pc = 8 * (int)ldw;   // bytes of 8 rows
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  // the load cursor: step l_step of the sequence's tile l_it, and the lane offsets of that step
  u32x4 ad{}, wd{};
  int l_it = 0, l_step = 0;
  int a_at[2], w_at[2];
  auto set_tile = [&](int it) {
    if (it < seq.count) {
      int tm, tn;
      seq.coords(it, tm, tn);
      ad = make_desc(A + (int64_t)tm * BM * lda, min((int64_t)0x7FFFFFFF, (int64_t)(M - tm * BM - 1) * lda + K));
      wd = make_desc(W + (int64_t)tn * BN * ldw, min((int64_t)0x7FFFFFFF, (int64_t)(N - tn * BN - 1) * ldw + K));
    } else {   // past the last tile: empty ranges
      ad[2] = 0;
      wd[2] = 0;
    }
  };
  auto set_step = [&] {
    const int last = l_step == KT - 1 ? -1 : 0;
#pragma unroll
    for (int par = 0; par < 2; ++par) {   // offsets of rows are below 2^30
      a_at[par] = a_vo[par] | (behind[par] & last);
      w_at[par] = w_vo[par] | (behind[par] & last);
    }
  };
  auto advance = [&] {
    if (++l_step == KT) {
      l_step = 0;
      set_tile(++l_it);
    }
    set_step();
  };
  auto load_a = [&](int u, int slot) {
    load_lds16(ad, a_at[u & 1] + u * a_pc, l_step * BK, lds_base + slot * S::kSlotA + (LA * wave + u) * 1024);
  };
  auto load_w = [&](int u, int slot) {
    load_lds16(wd, w_at[u & 1] + u * w_pc, l_step * BK, lds_base + S::kBaseW + slot * S::kSlotW + (LW * wave + u) * 1024);
  };
  auto load_x = [&](int u, int slot) { if (XA) load_a(u, slot); else load_w(u, slot); };
  auto load_y = [&](int u, int slot) { if (XA) load_w(u, slot); else load_a(u, slot); };

  // ---- fragment reads: row base + 16 b + (lane & 15), logical chunk 4 kk + (lane >> 4) of half kk
  const int fr = lane & 15, fh = lane >> 4;
  const int sw = row_swizzle(fr);   // == row_swizzle(base + 16 b + fr)
  int fo_a[2], fo_w[2];             // + 16 * kRowBytes b
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    fo_a[kk] = (wm * 16 * MB + fr) * kRowBytes + (((4 * kk + fh) ^ sw) << 4);
    fo_w[kk] = S::kBaseW + (wn * 16 * NB + fr) * kRowBytes + (((4 * kk + fh) ^ sw) << 4);
  }
  struct Frags { i32x4 w[NB], a[MB]; };
  Frags f0, f1;
  // acc[i][j][e] = sum of row m, column n, m = 16 MB wm + 16 j + fr and n = 16 NB wn + 16 i + 4 fh + e of the tile
  i32x4 acc[NB][MB];

  // One half: the MFMAs on f, each followed by its share of the reads of the
  // next half into g and of the loads, fenced so that the compiler keeps this order.
  constexpr int NM = MB * NB, NR = MB + NB;
  constexpr int kReadStep = 2, kLoadStep = NM >= 48 ? 4 : 2;
  static_assert((NM - 1) / kReadStep + 1 >= NR && (NM - 1) / kLoadStep + 1 >= (LX > LY ? LX : LY), "all reads and loads are issued");
  auto half = [&](const Frags& f, Frags& g, int slot_x, int slot_y, int kk, auto loads_x, int load_slot) __attribute__((always_inline)) {
    constexpr bool kX = decltype(loads_x)::value;
    const char* const pa = smem + (XA ? slot_x : slot_y) * S::kSlotA + fo_a[kk];
    const char* const pw = smem + (XA ? slot_y : slot_x) * S::kSlotW + fo_w[kk];
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      const int i = m / MB, j = m % MB;
      mfma16(acc[i][j], f.w[i], f.a[j]);
      const int r = m / kReadStep;   // reads in the order of their use: w0, a0 .., w1 ..
      if (m % kReadStep == 0 && r < NR) {
        if (r == 0) g.w[0] = *reinterpret_cast<const i32x4*>(pw);
        else if (r <= MB) g.a[r - 1] = *reinterpret_cast<const i32x4*>(pa + (r - 1) * 16 * kRowBytes);
        else g.w[r - MB] = *reinterpret_cast<const i32x4*>(pw + (r - MB) * 16 * kRowBytes);
      }
      const int l = m / kLoadStep;
      if (m % kLoadStep == 0 && l < (kX ? LX : LY)) {
        if (kX) load_x(l, load_slot);
        else load_y(l, load_slot);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // the first tile's steps 0 .. R - 1, then the fragments of step 0's first half
  set_tile(0);
  set_step();
#pragma unroll
  for (int s = 0; s < RX; ++s) {
#pragma unroll
    for (int u = 0; u < LX; ++u) load_x(u, s);
#pragma unroll
    for (int u = 0; u < LY; ++u) load_y(u, s);
    advance();
  }
  wait_vmcnt<(RX - 1) * (LX + LY)>();
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NB; ++i) f0.w[i] = *reinterpret_cast<const i32x4*>(smem + fo_w[0] + i * 16 * kRowBytes);
#pragma unroll
  for (int j = 0; j < MB; ++j) f0.a[j] = *reinterpret_cast<const i32x4*>(smem + fo_a[0] + j * 16 * kRowBytes);
  int sx = 0, sy = 0;   // slots of the current step, counted over all tiles: mod RX, mod RY
  for (int it = 0; it < seq.count; ++it) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < MB; ++j) acc[i][j] = i32x4{};
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 1");   // a vector write of an MFMA's addend
    __builtin_amdgcn_sched_barrier(0);
    int tm, tn;
    seq.coords(it, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN;
    int last_y = 0;
    for (int s = 0; s < KT; ++s) {
      const int sx1 = sx == RX - 1 ? 0 : sx + 1;
      const int sy1 = sy == RY - 1 ? 0 : sy + 1;
      half(f0, f1, sx, sy, 1, std::false_type{}, sy == 0 ? RY - 1 : sy - 1);   // loads Y(s + R) into the slot of s - 1
      // X(s + 1) and Y(s + 1) have landed; R - 2 steps of X and R - 1 of Y may still be in flight
      wait_vmcnt<(RX - 2) * LX + (RX - 1) * LY>();
      __syncthreads();
      __builtin_amdgcn_sched_barrier(0);
      half(f1, f0, sx1, sy1, 0, std::true_type{}, sx);                         // loads X(s + R) into the slot of s
      advance();
      last_y = sy;
      sx = sx1;
      sy = sy1;
    }
    // wait states from the last MFMA to a vector read of its result (the compiler itself would put at most 12)
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);

    // Epilogue through a wave-private LDS window of 32 rows x CW columns
    // (fp32), in the part of the last step's Y slot that this wave itself
    // refills in the next step: the places, permutation and swizzle of the
    // bf16 kernel's.  What goes through the window is the sum times the row's
    // scale, which a lane of the MFMA layout needs one of per block.  One
    // wave's LDS operations complete in order, so the window needs no barrier.
    // out may be res: every element is read before it is written, by the same lane.
    constexpr int CW = NB % 4 == 0 && LY >= 8 ? 64 : 32;   // the wave's share of a Y slot is LY KiB
    constexpr int LPR = CW / 8, RPP = 64 / LPR;            // lanes per row and rows per pass when read back
    constexpr int NP = 32 / RPP, NV = NB * 16 / CW;        // passes per window, windows per row block pair
    static_assert(32 * CW * 4 <= LY * 1024 && NB * 16 % CW == 0 && MB % 2 == 0, "the window fits");
    constexpr bool kRes = EPI == DIT_EPI_RESIDUAL || EPI == DIT_EPI_GATED_RESIDUAL;
    constexpr int kAhead = sizeof(T) == 2 ? 1 : 0;         // row block pairs by which the residual is loaded ahead
    char* const ew = smem + (XA ? S::kBaseW + last_y * S::kSlotW : last_y * S::kSlotA) + wave * (LY * 1024);
    // The lane, hidden from the compiler: it would form the window's addresses
    // once before the tiles, and keep them in scratch memory meanwhile.
    int el = lane;
    asm volatile("" : "+v"(el));
    const int er = el / LPR, ec = el % LPR, wr = el & 15, wh = el >> 4;
    auto at = [](int r, int c) {   // LDS byte of chunk c of window row r
      if (CW == 64) return r * 256 + ((((c >> 1) | ((c & 1) << 3)) ^ (((r & 1) << 3) | ((r >> 1) & 7))) << 4);
      return r * 128 + ((((c >> 1) | ((c & 1) << 2)) ^ ((((r >> 1) & 1) << 2) | ((r >> 2) & 3))) << 4);
    };
    const int nw = n0 + wn * 16 * NB + 8 * ec;   // the lane's first column of window 0
    float row_scale[MB];
#pragma unroll
    for (int j = 0; j < MB; ++j) row_scale[j] = ep.sa[min(m0 + wm * 16 * MB + 16 * j + wr, M - 1)];
    float wscale[NV][8], bsum[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int n = nw + CW * v;
#pragma unroll
      for (int e = 0; e < 8; ++e) wscale[v][e] = bsum[v][e] = 0.f;
      if (n < N) {
#pragma unroll
        for (int e = 0; e < 8; ++e) wscale[v][e] = ep.sw[n + e];
        if (ep.bias) {
          const V8 bv = *reinterpret_cast<const V8*>(ep.bias + n);
#pragma unroll
          for (int e = 0; e < 8; ++e) bsum[v][e] = (float)bv[e];
        }
      }
    }
    V8 rv[1 + kAhead][NV][NP];
    auto load_res = [&](int j) __attribute__((always_inline)) {
      if constexpr (kRes) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const int m = m0 + wm * 16 * MB + 32 * j + RPP * p + er, n = nw + CW * v;
            rv[j & kAhead][v][p] = V8{};
            if (m < M && n < N) rv[j & kAhead][v][p] = *reinterpret_cast<const V8*>(ep.res + (int64_t)m * ep.ldr + n);
          }
      }
    };
    if (kAhead) load_res(0);
#pragma unroll
    for (int j = 0; j < MB / 2; ++j) {
      if (j + kAhead < MB / 2) load_res(j + kAhead);
      const int mb = m0 + wm * 16 * MB + 32 * j;   // first row of the pair
      f32x4 gv[NV][2];
      bool g_one = true;                           // all rows of the pair belong to one request
      if (EPI == DIT_EPI_GATED_RESIDUAL) {
        const int r_lo = find_req(ep.req.cu, ep.req.n_req, min(mb, M - 1));
        const int r_hi = find_req(ep.req.cu, ep.req.n_req, min(mb + 31, M - 1));
        g_one = r_lo == r_hi;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          gv[v][0] = gv[v][1] = f32x4{};
          if (g_one && nw + CW * v < N) {
            const float* gp = ep.gate + (int64_t)r_lo * ep.gate_stride + nw + CW * v;
            gv[v][0] = *reinterpret_cast<const f32x4*>(gp);
            gv[v][1] = *reinterpret_cast<const f32x4*>(gp + 4);
          }
        }
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int ii = 0; ii < CW / 16; ++ii)
#pragma unroll
          for (int jj = 0; jj < 2; ++jj) {
            const i32x4 c = acc[v * (CW / 16) + ii][2 * j + jj];
            f32x4 z;
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = (float)c[e] * row_scale[2 * j + jj];
            *reinterpret_cast<f32x4*>(ew + at(16 * jj + wr, 4 * ii + wh)) = z;
          }
        const int n = nw + CW * v;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const int r = RPP * p + er, m = mb + r;
          const f32x4 z0 = *reinterpret_cast<const f32x4*>(ew + at(r, 2 * ec));
          const f32x4 z1 = *reinterpret_cast<const f32x4*>(ew + at(r, 2 * ec + 1));
          float z[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = fmaf(e < 4 ? z0[e & 3] : z1[e & 3], wscale[v][e], bsum[v][e]);
          if (EPI == DIT_EPI_GELU_TANH) {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = gelu_tanh(z[e]);
          } else if (EPI == DIT_EPI_GATED_RESIDUAL) {
            f32x4 g0 = gv[v][0], g1 = gv[v][1];
            if (!g_one && m < M && n < N) {   // the pair spans a request boundary
              const float* gp = ep.gate + (int64_t)find_req(ep.req.cu, ep.req.n_req, m) * ep.gate_stride + n;
              g0 = *reinterpret_cast<const f32x4*>(gp);
              g1 = *reinterpret_cast<const f32x4*>(gp + 4);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = fmaf(e < 4 ? g0[e & 3] : g1[e & 3], z[e], (float)rv[j & kAhead][v][p][e]);
          } else if (EPI == DIT_EPI_RESIDUAL) {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = (float)rv[j & kAhead][v][p][e] + z[e];
          }
          V8 o;
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = (T)z[e];
          // computed on every path: were it left to the branch, a load above
          // would be pending where the branch is not taken, and the compiler
          // would wait for all loads in the K loop
          asm volatile("" : "+v"(o));
          if (m < M && n < N) *reinterpret_cast<V8*>(ep.out + (int64_t)m * ep.ldo + n) = o;
        }
      }
    }
    // the window's reads are done before the next step's loads overwrite it
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  wait_vmcnt<0>();   // no load may land in LDS after the workgroup has ended
}

// ---------------------------------------------------------------- few rows
//
// Up to 64 rows: a workgroup of 8 waves computes MB x NB blocks of 16 x 16 (all
// rows, 16 NB output channels), the waves share K in turns of 128 bytes and
// their sums, whole numbers, meet in LDS.  The operands go from global memory
// straight into the matrix instruction's registers: 16 rows x 64 bytes a load.
// Bound by the weights, which are read once.
constexpr int kFewWaves = 8;

template <typename T, int EPI, int MB, int NB>
__global__ __launch_bounds__(64 * kFewWaves) void gemm_i8_few(
    const int8_t* __restrict__ A, int64_t lda, const int8_t* __restrict__ W, int64_t ldw, Epi<T> ep, int M, int N, int K) {
  typedef T V4 __attribute__((ext_vector_type(4)));
  constexpr int U = MB * NB <= 2 ? 5 : MB * NB <= 4 ? 3 : 2;   // turns in flight
  __shared__ i32x4 part[kFewWaves][MB * NB][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fh = lane >> 4;
  const int n0 = blockIdx.x * 16 * NB, m0 = blockIdx.y * 16 * MB;
  const int8_t *pa[MB], *pw[NB];   // rows past the last repeat it
#pragma unroll
  for (int j = 0; j < MB; ++j) pa[j] = A + (int64_t)min(m0 + 16 * j + fr, M - 1) * lda + 16 * fh;
#pragma unroll
  for (int i = 0; i < NB; ++i) pw[i] = W + (int64_t)min(n0 + 16 * i + fr, N - 1) * ldw + 16 * fh;
  i32x4 acc[NB][MB] = {};
  struct Step { i32x4 a[MB][2], w[NB][2]; };
  // the turn from byte k on: FULL, or what K leaves of it (a lane's 16 bytes are inside or outside)
  auto load = [&](Step& s, int k, auto full) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool in = decltype(full)::value || k + 64 * h + 16 * fh < K;
#pragma unroll
      for (int i = 0; i < NB; ++i) s.w[i][h] = in ? *reinterpret_cast<const i32x4*>(pw[i] + k + 64 * h) : i32x4{};
#pragma unroll
      for (int j = 0; j < MB; ++j) s.a[j][h] = in ? *reinterpret_cast<const i32x4*>(pa[j] + k + 64 * h) : i32x4{};
    }
  };
  auto mma = [&](const Step& s) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(s.w[i][h], s.a[j][h], acc[i][j], 0, 0, 0);
  };
  const int whole = K / BK;   // whole turns; wave w takes turns w, w + 8, ..
  int t = wave;
  for (; t + kFewWaves * (U - 1) < whole; t += kFewWaves * U) {
    Step s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) load(s[u], (t + kFewWaves * u) * BK, std::true_type{});
#pragma unroll
    for (int u = 0; u < U; ++u) mma(s[u]);
  }
  if (t * BK < K) {   // up to U turns more, the last one perhaps not whole
    Step s[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if ((t + kFewWaves * u) * BK < K) load(s[u], (t + kFewWaves * u) * BK, std::false_type{});
#pragma unroll
    for (int u = 0; u < U; ++u)
      if ((t + kFewWaves * u) * BK < K) mma(s[u]);
  }
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j) part[wave][i * MB + j][lane] = acc[i][j];
  __syncthreads();
  for (int b = wave; b < MB * NB; b += kFewWaves) {
    i32x4 c = part[0][b][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) c += part[w][b][lane];
    const int m = m0 + 16 * (b % MB) + fr, n = n0 + 16 * (b / MB) + 4 * fh;
    if (m >= M || n >= N) continue;
    const float sa = ep.sa[m];
    float z[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = fmaf((float)c[e] * sa, ep.sw[n + e], ep.bias ? (float)ep.bias[n + e] : 0.f);
    if (EPI == DIT_EPI_GELU_TANH) {
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = gelu_tanh(z[e]);
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
}

// -------------------------------------------------------------- the choice

// The tile shapes, by the index of kCost.
typedef Shape<8, 8, 2, false> Tile256x256;
typedef Shape<8, 6, 2, false> Tile256x192;
typedef Shape<4, 8, 2, true> Tile128x256;
typedef Shape<4, 6, 3, false> Tile128x192;
typedef Shape<4, 4, 4, false> Tile128x128;
struct TileCost { int bm, bn; float fixed, step, full; };
constexpr TileCost kCost[5] = {
    {256, 256, 7.15f, 0.9445f, 0.3357f}, {256, 192, 5.97f, 0.7277f, 0.2706f}, {128, 256, 4.45f, 0.5556f, 0.1872f},
    {128, 192, 3.34f, 0.4396f, 0.1457f}, {128, 128, 2.74f, 0.3213f, 0.1101f}};
constexpr int kFew = 5;   // the index of the kernel for few rows
constexpr int kFewRows = 64;
constexpr int kFewColumns = 1 << 24;   // 512 work-items for 16 channels: 2^29 in the launch's first dimension
int few_tile_m(int64_t M) { return M <= 16 ? 16 : M <= 32 ? 32 : 64; }

std::atomic<int> g_shape{-1};   // forced shape (-1: chosen per call)

int choose(int64_t M, int N, int K, int cus) {
  const bool few = M <= 64 * kFewRows && N <= kFewColumns;   // what the launch of that kernel holds
  const int forced = g_shape.load(std::memory_order_relaxed);
  if (forced >= 0 && (forced != kFew || few)) return forced;
  if (few && M <= kFewRows) return kFew;
  const float kt = (float)((K + BK - 1) / BK);
  int best = 0;
  float least = 0.f;
  for (int t = 0; t < 5; ++t) {
    const TileCost& c = kCost[t];
    const int64_t tiles = ((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn);
    const int64_t rounds = tiles / cus, rest = tiles % cus;
    const float cost = (float)rounds * (c.fixed + kt * (c.step + c.full)) +
                       (rest ? c.fixed + kt * (c.step + c.full * (float)rest / (float)cus) : 0.f);
    if (t == 0 || cost < least) {
      best = t;
      least = cost;
    }
  }
  return best;
}

// Tile rows per raster group, as for the bf16 kernel.
int raster(int tiles_m) { return tiles_m <= 40 ? 8 : tiles_m <= 160 ? 4 : 3; }

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
                                                  (int)tiles_n, raster((int)tiles_m));
  return hipGetLastError();
}

template <typename T, int EPI, int MB, int NB>
hipError_t launch_few(const LinearI8Args& p, hipStream_t s) {
  const dim3 grid((unsigned)((p.N + 16 * NB - 1) / (16 * NB)), (unsigned)((p.M + 16 * MB - 1) / (16 * MB)));
  gemm_i8_few<T, EPI, MB, NB><<<grid, 64 * kFewWaves, 0, s>>>(p.a, p.lda, p.w, p.ldw, epi_of<T>(p), (int)p.M, p.N, p.K);
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
    default: break;
  }
  switch (few_tile_m(p.M)) {
    case 16: return launch_few<T, EPI, 1, 1>(p, s);
    case 32: return launch_few<T, EPI, 2, 1>(p, s);
    default: return launch_few<T, EPI, 4, 1>(p, s);
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
  int shape = tile_m == 0 && tile_n == 0 ? -1 : tile_m == 16 && tile_n == 16 ? kFew : -2;
  for (int t = 0; t < 5; ++t)
    if (kCost[t].bm == tile_m && kCost[t].bn == tile_n) shape = t;
  if (shape >= -1) g_shape.store(shape, std::memory_order_relaxed);
  return shape >= -1;
}

void linear_i8_plan(int64_t M, int N, int K, int cus, int* tile_m, int* tile_n) {
  const int t = choose(M, N, K, cus);
  *tile_m = t == kFew ? few_tile_m(M) : kCost[t].bm;
  *tile_n = t == kFew ? 16 : kCost[t].bn;
}

hipError_t launch_linear_i8(const LinearI8Args& p, hipStream_t s) {
  if (p.M == 0) return hipSuccess;
  return p.dtype == DIT_BF16 ? launch_typed<bf16>(p, s) : launch_typed<float>(p, s);
}

}  // namespace dit
