// Attention over the paged 8-bit key/value cache: O = softmax(q k^T scale) v
// for the packed queries of each request over its cached tokens, no mask.
//
// Rows.  The query heads that share a key/value head are rows of one matrix:
// row i of (request, key/value head) is token i / G, query head i % G of the
// group of G heads.
//
// The tokens of a page lie in groups of 32 in the order of the matrix
// instructions' operands, so every operand is read as 16 contiguous bytes per
// lane, from LDS without bank conflicts and from global memory as whole KiB:
//   keys   [head_dim / 16][32 tokens][16 channels]
//   values [2][head_dim][16 tokens: 4 i + j <-> token 8 i + 4 f + j]
//
// S^T = K Q^T in bf16.  The keys' codes go to v_mfma_scale_f32_32x32x64_f8f6f4
// as they are stored, with the page's scale byte as the instruction's block
// scale.  A bf16 query value has 8 significant bits, two e4m3 values 4 each:
// q = q1 + q2 exactly (values below 2^-15 of the largest of their 64 channels
// to 2^-23 of it), so two of the fp8 instructions, at twice the bf16 rate,
// give what a bf16 product of converted keys would, without the conversion.
// O^T = V^T P^T in bf16 MFMAs: v_cvt_scalef32_pk_bf16_fp8 turns two codes into
// bf16 with the page's scale, exactly.
//
// Softmax is fp32 in log2 units: a score is multiplied by scale * log2(e) in
// the multiply-add that takes off the row's reference.  (Multiplied into the
// query instead, it would have to be rounded to bf16 with it: the output was
// then 0.0037 off the exact one, root mean square, 0.0017 of which is its own
// rounding; now 0.0024.)  Probabilities are rounded to bf16, 8 significant bits
// each, and their sum is that of the rounded ones.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace dit {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kXcds = 8;

// What the kernels need besides the caller's arguments: the row tiles of the
// requests that have queries.  An item is (request, key/value head, key piece,
// row tile), numbered with the row tiles of a head and piece side by side.
struct CachedWork {
  int n_req, pieces;
  int n_pages, page_shift, max_pages, max_len;
  int n_heads, n_kv_heads, group;   // group: query heads of a key/value head
  int64_t q_stride, o_stride;
  const char *k_pages, *v_pages;
  const uint8_t *k_scale, *v_scale;
  const int32_t *table, *lens;
  const bf16* q_gain;
  float q_eps, scale_log2;
  float* part;                      // pieces > 1: fp32 [pieces][rows][head_dim], then [pieces][rows][2]
  int64_t part_rows;                // tokens * n_heads
  int req[DIT_MAX_REQ];             // the request's index (its row of the table)
  int q_start[DIT_MAX_REQ];
  int q_len[DIT_MAX_REQ];
  int tiles[DIT_MAX_REQ];
  int prefix[DIT_MAX_REQ + 1];      // items before request i
};

struct Item {
  int i, head, piece, tile;   // position in the work table, key/value head, key piece, row tile
};

// Workgroups are dispatched to the XCDs round-robin: each XCD takes the same
// contiguous eighth of every request's items, so the row tiles that read the
// same keys stay on one XCD and share its L2.
__device__ __forceinline__ bool find_item(const CachedWork& w, Item& it) {
  const int xcd = blockIdx.x % kXcds;
  int j = blockIdx.x / kXcds;
  for (int r = 0; r < w.n_req; ++r) {
    const int n = w.prefix[r + 1] - w.prefix[r];
    const int lo = (int)((int64_t)xcd * n / kXcds), hi = (int)((int64_t)(xcd + 1) * n / kXcds);
    if (j < hi - lo) {
      const int local = lo + j;
      const int hp = local / w.tiles[r];
      it.i = r;
      it.tile = local - hp * w.tiles[r];
      it.head = hp / w.pieces;
      it.piece = hp - it.head * w.pieces;
      return true;
    }
    j -= hi - lo;
  }
  return false;
}

// The request's cached length, within the table and the caller's bound.
__device__ __forceinline__ int length_of(const CachedWork& w, int r) { return min(max(w.lens[r], 0), w.max_len); }

// Position of a group of 32 tokens in the pool, in groups (its page, head and
// place in the page), and its two scale bytes; none where the table names no
// page of the pool.
constexpr uint32_t kNoGroup = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t find_group(const CachedWork& w, int r, int head, int g, uint32_t& scales) {
  const int gs = w.page_shift - 5;   // log2 groups per page
  const int page = w.table[(int64_t)r * w.max_pages + (g >> gs)];
  scales = 0x7F7Fu;
  if (page < 0 || page >= w.n_pages) return kNoGroup;
  const uint32_t slot = (uint32_t)page * w.n_kv_heads + head;
  scales = w.k_scale[slot] | (uint32_t)w.v_scale[slot] << 8;
  return (slot << gs) + (g & ((1 << gs) - 1));
}

__device__ __forceinline__ float pow2(uint32_t biased) { return __uint_as_float(biased << 23); }

// This lane's query row as the B operand of S^T: channels 64 c + 32 h + 16 f
// .. +15 of the row (f: the lane's half; h: 0, 1), with QNORM RMS-normalised and
// rounded to bf16, split into two e4m3 parts with one power of two per row and 64 channels (the
// same byte in both lanes of a row: the instruction's blocks of 32 channels each
// span both).
template <int HD> struct QFrag {
  i32x8 hi[HD / 64], lo[HD / 64];
  int scales;   // byte 2 c: of hi[c], byte 2 c + 1: of lo[c] (smaller by 2^-4)
};

template <int HD, bool QNORM>
__device__ __forceinline__ void load_query(const bf16* row, int f, const CachedWork& w, QFrag<HD>& q) {
  constexpr int NC = HD / 64;
  bf16x8 raw[4 * NC];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        raw[4 * c + 2 * h + k] = *reinterpret_cast<const bf16x8*>(row + 64 * c + 32 * h + 16 * f + 8 * k);
  float mul = 1.f;
  bf16x8 gain[QNORM ? 4 * NC : 1];
  if constexpr (QNORM) {
    // RMSNorm over the head: this lane holds half of its values, the lane 32 apart the other half
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * NC; ++i) {
      gain[i] = *reinterpret_cast<const bf16x8*>(w.q_gain + 64 * (i / 4) + 32 * (i / 2 % 2) + 16 * f + 8 * (i % 2));
      const f32x8 x = __builtin_convertvector(raw[i], f32x8);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
    }
    ss += __shfl_xor(ss, 32, kWave);
    mul = rsqrtf(ss * (1.0f / HD) + w.q_eps);
  }
  uint32_t bytes = 0;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float x[32];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x8 v = __builtin_convertvector(raw[4 * c + i], f32x8);
      if constexpr (QNORM) v = v * mul * __builtin_convertvector(gain[4 * c + i], f32x8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[8 * i + e] = (float)(bf16)v[e];
        const uint32_t u = __float_as_uint(x[8 * i + e]) & 0x7FFFFFFFu;
        if (u < 0x7F800000u) top = max(top, u);
        else x[8 * i + e] = __uint_as_float(0x7FC00000u);   // an infinity has no code: NaN
      }
    }
    // smallest power of two with every value of the row's 64 channels (this
    // lane's and the lane's 32 apart) below 448 of it; 16 and more, so that the
    // low part's byte stays positive
    top = max(top, (uint32_t)__shfl_xor((int)top, 32, kWave));
    const uint32_t s = (uint32_t)max((int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u), 16);
    bytes |= (s | (s - 4) << 8) << (16 * c);
    const float inv = pow2(254 - s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float a[4], b[4];
      int hw = 0, lw = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = x[4 * i + e] * inv;
      hw = __builtin_amdgcn_cvt_pk_fp8_f32(a[0], a[1], hw, false);
      hw = __builtin_amdgcn_cvt_pk_fp8_f32(a[2], a[3], hw, true);
      const f32x2 r0 = __builtin_amdgcn_cvt_pk_f32_fp8(hw, false), r1 = __builtin_amdgcn_cvt_pk_f32_fp8(hw, true);
      b[0] = (a[0] - r0[0]) * 16.f;
      b[1] = (a[1] - r0[1]) * 16.f;
      b[2] = (a[2] - r1[0]) * 16.f;
      b[3] = (a[3] - r1[1]) * 16.f;
      lw = __builtin_amdgcn_cvt_pk_fp8_f32(b[0], b[1], lw, false);
      lw = __builtin_amdgcn_cvt_pk_fp8_f32(b[2], b[3], lw, true);
      q.hi[c][i] = hw;
      q.lo[c][i] = lw;
    }
  }
  q.scales = (int)bytes;
}

// acc += K Q^T for one 64-channel step C: a[0], a[1] are the lane's two
// 16-byte key pieces (key lane % 32), ks the scale byte of the group's keys
template <int C, int HD>
__device__ __forceinline__ f32x16 score_step(const u32x4& a0, const u32x4& a1, const QFrag<HD>& q, int ks, f32x16 acc) {
  const i32x8 a = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
  acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q.hi[C], acc, 0, 0, 0, ks, 2 * C, q.scales);
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q.lo[C], acc, 0, 0, 0, ks, 2 * C + 1, q.scales);
}

// 8 codes (two dwords) of one value channel -> bf16 with the page's scale
__device__ __forceinline__ bf16x8 values8(uint32_t w0, uint32_t w1, float vs) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, vs, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, vs, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, vs, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, vs, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// acc + a[0] + a[1]
__device__ __forceinline__ float add_pair(bf16x2 a, float acc) {
  return __builtin_amdgcn_fdot2_f32_bf16(a, bf16x2{(bf16)1.f, (bf16)1.f}, acc, false);
}

// Bytes of tokens 8 i + 4 f + 0 .. 3 of a group that are among its first n.
// Codes past the request's end are whatever the page held before, NaN among
// them, which a probability of 0 would not take out of the product.
__device__ __forceinline__ uint32_t token_mask(int i, int f, int n) {
  const int left = n - 8 * i - 4 * f;
  return left >= 4 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
}

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// 16 bytes per lane from global memory straight into LDS bytes lds + OFF +
// 16 lane .. +15; completion is tracked by hand (wait_vmcnt) and published by
// the workgroup barrier.  Loads past the descriptor's record count give zeros.
template <uint32_t OFF>
__device__ __forceinline__ void load_lds16(const u32x4& desc, uint32_t voff, uint32_t lds) {
  asm volatile("s_add_u32 m0, %0, %3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(lds), "v"(voff), "s"(desc), "n"(OFF) : "m0", "scc");
}
#pragma clang diagnostic pop
template <int N> __device__ __forceinline__ void wait_vmcnt() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N)); }

// ------------------------------------------------- bf16, many rows of a head

constexpr int kChunkTiles = 512;      // 64-token tiles whose groups are looked up at once (8 KB of LDS)
constexpr float kHeadroom = 18446744073709551616.0f;   // 2^64, bound of a row sum

// 4 waves of 32 rows; tiles of 64 tokens (8 KB of keys and 8 KB of values at
// 128 channels: half of bf16) in an LDS ring of 4, loaded three tiles ahead;
// two workgroups per compute unit.
//
// The row reference of the softmax is the first tile's row maximum for the
// whole pass, so the loop neither searches maxima nor rescales the output.
// Where a row's sum passes 2^64 the workgroup finds the exact maxima and runs
// again, so the result is the softmax in any case.
template <int HD, bool QNORM>
__global__ __launch_bounds__(256, 2) void cached_attn_many(const bf16* __restrict__ Q, bf16* __restrict__ O,
                                                           CachedWork w) {
  constexpr int NC = HD / 64;          // matrix instructions over the channels
  constexpr int ND = HD / 32;          // 32-channel blocks of the output
  constexpr int kGroup = 32 * HD;      // bytes of a group's keys
  constexpr int kSlot = 4 * kGroup;    // a tile: keys of both groups, then values of both
  constexpr int kLoads = kSlot / 4096; // 1 KB loads per wave and tile
  constexpr int kRing = 4;
  __shared__ __attribute__((aligned(1024))) char smem[kRing * kSlot];
  __shared__ u32x2 groups[2 * kChunkTiles];   // position in the pool, scale bytes
  __shared__ int s_bad, s_redo;

  Item it;
  if (!find_item(w, it)) return;
  const int r = w.req[it.i];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fr = lane & 31, fh = lane >> 5;
  const int rows = w.q_len[it.i] * w.group;
  const int my_row = it.tile * 128 + wave * 32 + fr;
  const int row = min(my_row, rows - 1);
  const int token = w.q_start[it.i] + row / w.group;
  const int q_head = it.head * w.group + row % w.group;

  const int len = length_of(w, r);
  const int all_tiles = (len + 63) / 64;
  const int per = (all_tiles + w.pieces - 1) / w.pieces;
  const int t_begin = min(it.piece * per, all_tiles), t_end = min(t_begin + per, all_tiles);

  QFrag<HD> q;
  load_query<HD, QNORM>(Q + (int64_t)token * w.q_stride + q_head * HD, fh, w, q);

  const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_char*)smem;
  const uint32_t voff = (uint32_t)(wave * 1024 % kGroup + lane * 16);
  int chunk0 = 0;   // first tile of the groups in LDS
  auto issue = [&](int t) __attribute__((always_inline)) {
    const uint32_t lds = lds_base + (uint32_t)((t % kRing) * kSlot + wave * 1024);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int part = (wave + 4 * u) * 1024 / kGroup;   // 0, 1: keys of the groups; 2, 3: values
      const uint32_t g = __builtin_amdgcn_readfirstlane(groups[2 * (t - chunk0) + (part & 1)][0]);
      const uint64_t base = (uint64_t)(uintptr_t)(part >> 1 ? w.v_pages : w.k_pages) + (uint64_t)(g == kNoGroup ? 0u : g) * kGroup;
      const u32x4 desc = {(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, g == kNoGroup ? 0u : (uint32_t)kGroup, 0x00020000u};
      if (u == 0) load_lds16<0>(desc, voff, lds);
      else if (u == 1) load_lds16<4096>(desc, voff, lds);
      else if (u == 2) load_lds16<8192>(desc, voff, lds);
      else load_lds16<12288>(desc, voff, lds);
    }
  };

  f32x16 oacc[ND];
  float l_run[2];
  float m_ref = 0.f, x_max = -INFINITY;
  bool have_ref = false;
  const float c = w.scale_log2;
  const float off_score = c < 0.f ? INFINITY : -INFINITY;   // times c: -inf

  // One tile.  MASKED (its codes of values are then clean, see run_pass): n[hb]
  // tokens of each group count; track: only the largest score is wanted.
  auto tile = [&](int t, bool masked, int n0, int n1, bool track) __attribute__((always_inline)) {
    const char* slot = smem + (t % kRing) * kSlot;
    const u32x2 d0 = groups[2 * (t - chunk0)], d1 = groups[2 * (t - chunk0) + 1];
    f32x16 s[2];
#pragma unroll
    for (int hb = 0; hb < 2; ++hb) {
      const int ks = (int)(hb ? d1[1] : d0[1]);
      const u32x4* kp = reinterpret_cast<const u32x4*>(slot + hb * kGroup) + lane;
      s[hb] = score_step<0, HD>(kp[0], kp[64], q, ks, f32x16{});
      if constexpr (NC == 2) s[hb] = score_step<1, HD>(kp[128], kp[192], q, ks, s[hb]);
    }
    if (masked) {
#pragma unroll
      for (int hb = 0; hb < 2; ++hb)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (8 * (v >> 2) + 4 * fh + (v & 3) >= (hb ? n1 : n0)) s[hb][v] = off_score;
    }
    if (track || !have_ref) {
      float mx = -INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, fmaxf(s[0][v] * c, s[1][v] * c));
      if (track) {
        x_max = fmaxf(x_max, mx);
        return;
      }
      m_ref = fmaxf(mx, __shfl_xor(mx, 32, kWave));
      have_ref = true;
    }
    bf16x8 p[4];
#pragma unroll
    for (int hb = 0; hb < 2; ++hb)
#pragma unroll
      for (int v = 0; v < 16; v += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[hb][v], c, -m_ref));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[hb][v + 1], c, -m_ref));
        const bf16x2 pr = __builtin_convertvector((f32x2){p0, p1}, bf16x2);
        p[2 * hb + (v >> 3)][v & 7] = pr[0];
        p[2 * hb + (v >> 3)][(v & 7) + 1] = pr[1];
        l_run[hb] = add_pair(pr, l_run[hb]);
      }
#pragma unroll
    for (int hb = 0; hb < 2; ++hb) {
      const float vs = pow2((hb ? d1[1] : d0[1]) >> 8);
      const u32x4* vp = reinterpret_cast<const u32x4*>(slot + (2 + hb) * kGroup + fh * (HD * 16)) + fr;
#pragma unroll
      for (int db = 0; db < ND; ++db) {
        const u32x4 x = vp[32 * db];
        oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8(x[0], x[1], vs), p[2 * hb], oacc[db], 0, 0, 0);
        oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8(x[2], x[3], vs), p[2 * hb + 1], oacc[db], 0, 0, 0);
      }
    }
  };

  auto run_pass = [&](bool track) __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < ND; ++db) oacc[db] = f32x16{};
    l_run[0] = l_run[1] = 0.f;
    for (int c0 = t_begin; c0 < t_end; c0 += kChunkTiles) {
      const int c1 = min(c0 + kChunkTiles, t_end);
      __syncthreads();   // the previous chunk's groups and tiles have been read
      if (tid == 0) s_bad = 0;
      __syncthreads();
      bool bad = false;
      for (int g = 2 * c0 + tid; g < 2 * c1; g += 256) {
        uint32_t scales = 0x7F7Fu, at = kNoGroup;
        if (32 * g < len) {
          at = find_group(w, r, it.head, g, scales);
          bad |= at == kNoGroup;
        }
        groups[g - 2 * c0] = u32x2{at, scales};
      }
      if (bad) s_bad = 1;
      __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): only tile loads are counted below
      __syncthreads();
      chunk0 = c0;
      const bool any_bad = __builtin_amdgcn_readfirstlane(s_bad) != 0;
      const int n_pre = min(3, c1 - c0);
      for (int t = 0; t < n_pre; ++t) issue(c0 + t);
      if (n_pre == 3) wait_vmcnt<2 * kLoads>();
      else if (n_pre == 2) wait_vmcnt<kLoads>();
      else wait_vmcnt<0>();
      __syncthreads();
      for (int t = c0; t < c1; ++t) {
        // a tile that ends early or lacks a page: the workgroup clears the value
        // codes of the tokens that do not count (whatever the page held before,
        // NaN among them, which a probability of 0 would not take out of the product)
        const bool masked = any_bad || 64 * (t + 1) > len;
        int n0 = 32, n1 = 32;
        if (masked) {
          const uint32_t g0 = groups[2 * (t - chunk0)][0], g1 = groups[2 * (t - chunk0) + 1][0];
          n0 = __builtin_amdgcn_readfirstlane(g0) == kNoGroup ? 0 : min(max(len - 64 * t, 0), 32);
          n1 = __builtin_amdgcn_readfirstlane(g1) == kNoGroup ? 0 : min(max(len - 64 * t - 32, 0), 32);
          u32x4* vals = reinterpret_cast<u32x4*>(smem + (t % kRing) * kSlot + 2 * kGroup);
#pragma unroll
          for (int e = tid; e < 4 * HD; e += 256) {
            const int f = e / HD % 2, n = e / HD < 2 ? n0 : n1;
            u32x4 x = vals[e];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] &= token_mask(i, f, n);
            vals[e] = x;
          }
          __syncthreads();
        }
        if (n0 + n1 > 0) tile(t, masked, n0, n1, track);   // (nothing there: the reference waits for the next tile)
        if (t + 1 < c1) {
          // tile t + 1 in LDS for every wave; tile t + 3 into the slot of t - 1
          if (t + 2 < c1) wait_vmcnt<kLoads>();
          else wait_vmcnt<0>();
          __syncthreads();
          if (t + 3 < c1) issue(t + 3);
        }
      }
    }
  };

  // The first pass against the first tile's maxima; where a row sum passed 2^64
  // (or overflowed), one to find the exact maxima and one against them.
  float l_tot = 0.f;
#pragma unroll 1
  for (int pass = 0;; ++pass) {
    run_pass(pass == 1);
    if (pass == 1) {
      m_ref = fmaxf(x_max, __shfl_xor(x_max, 32, kWave));
      continue;
    }
    const float l = l_run[0] + l_run[1];
    l_tot = l + __shfl_xor(l, 32, kWave);
    if (pass == 2) break;
    if (tid == 0) s_redo = 0;
    __syncthreads();
    if (__builtin_amdgcn_ballot_w64(!(l_tot <= kHeadroom)) != 0 && lane == 0) s_redo = 1;
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(s_redo) == 0) break;
  }

  // oacc[db][4 i + j]: channel 32 db + 8 i + 4 fh + j of the lane's row
  if (my_row >= rows) return;
  if (w.pieces > 1) {
    const int64_t id = (int64_t)it.piece * w.part_rows + (int64_t)token * w.n_heads + q_head;
    float* po = w.part + id * HD + 4 * fh;
#pragma unroll
    for (int db = 0; db < ND; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(po + 32 * db + 8 * i) =
            f32x4{oacc[db][4 * i], oacc[db][4 * i + 1], oacc[db][4 * i + 2], oacc[db][4 * i + 3]};
    if (fh == 0) *reinterpret_cast<f32x2*>(w.part + w.pieces * w.part_rows * HD + 2 * id) = f32x2{m_ref, l_tot};
    return;
  }
  const float inv = l_tot != 0.f ? 1.0f / l_tot : 0.f;   // no keys: a row of zeros
  bf16* op = O + (int64_t)token * w.o_stride + q_head * HD + 4 * fh;
#pragma unroll
  for (int db = 0; db < ND; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x4 ov;
#pragma unroll
      for (int j = 0; j < 4; ++j) ov[j] = (bf16)(oacc[db][4 * i + j] * inv);
      *reinterpret_cast<bf16x4*>(op + 32 * db + 8 * i) = ov;
    }
}

// ------------------------------------------------ the waves' shares, joined

// Row `row` of a workgroup's tile: WAVES partial outputs o[wave][channel][row],
// references m and sums l (log2 units; l 0: no keys), joined in wave order, then
// written to the output or, with more than one key piece, to the piece's part.
template <int HD, int ROWS, int WAVES, typename T>
__device__ __forceinline__ void join_waves(const float (&o)[WAVES][HD][ROWS + 1], const float (&m)[WAVES][ROWS],
                                           const float (&l)[WAVES][ROWS], int row0, int rows, const Item& it,
                                           const CachedWork& w, T* O) {
  for (int e = threadIdx.x; e < min(ROWS, rows - row0) * HD; e += WAVES * kWave) {
    const int i = e / HD, d = e % HD;
    const int row = row0 + i;
    const int token = w.q_start[it.i] + row / w.group;
    const int q_head = it.head * w.group + row % w.group;
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < WAVES; ++v)
      if (l[v][i] != 0.f) top = fmaxf(top, m[v][i]);
    float sum = 0.f, acc = 0.f;
#pragma unroll
    for (int v = 0; v < WAVES; ++v)
      if (l[v][i] != 0.f) {
        const float a = exp2f(m[v][i] - top);
        sum = fmaf(a, l[v][i], sum);
        acc = fmaf(a, o[v][d][i], acc);
      }
    if (w.pieces > 1) {
      const int64_t id = (int64_t)it.piece * w.part_rows + (int64_t)token * w.n_heads + q_head;
      w.part[id * HD + d] = acc;
      if (d == 0) *reinterpret_cast<f32x2*>(w.part + w.pieces * w.part_rows * HD + 2 * id) = f32x2{top, sum};
    } else {
      O[(int64_t)token * w.o_stride + q_head * HD + d] = from_f<T>(sum != 0.f ? acc / sum : 0.f);
    }
  }
}

// -------------------------------------------------- bf16, few rows of a head

// At most 32 rows per head: the cache is read once and bounds the time, so the
// waves share the tokens, not the rows.  Each wave takes every 4th group of 32
// tokens of its piece, straight from global memory into registers in the
// operands' order (whole KiB per load), two groups ahead, with an exact online
// softmax; the waves meet in LDS, the pieces in cached_attn_merge.
template <int HD, bool QNORM>
__global__ __launch_bounds__(256, 2) void cached_attn_few(const bf16* __restrict__ Q, bf16* __restrict__ O, CachedWork w) {
  constexpr int NC = HD / 64, ND = HD / 32, kGroup = 32 * HD, WAVES = 4;
  __shared__ float part_o[WAVES][HD][33];
  __shared__ float part_m[WAVES][32], part_l[WAVES][32];
  Item it;
  if (!find_item(w, it)) return;
  const int r = w.req[it.i];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fr = lane & 31, fh = lane >> 5;
  const int rows = w.q_len[it.i] * w.group;
  const int row = min(fr, rows - 1);
  const int token = w.q_start[it.i] + row / w.group;

  const int len = length_of(w, r);
  const int all = (len + 31) / 32;
  const int per = (all + w.pieces - 1) / w.pieces;
  const int g_begin = min(it.piece * per, all), g_end = min(g_begin + per, all);
  const int n_mine = max(0, (g_end - g_begin - wave + WAVES - 1) / WAVES);   // groups g_begin + wave + 4 i

  QFrag<HD> q;
  load_query<HD, QNORM>(Q + (int64_t)token * w.q_stride + (it.head * w.group + row % w.group) * HD, fh, w, q);

  uint32_t at = kNoGroup, scales = 0;   // lane i: this wave's group base + i
  int base = 0;
  auto look_up = [&](int i0) __attribute__((always_inline)) {
    base = i0;
    at = kNoGroup;
    if (i0 + lane < n_mine) at = find_group(w, r, it.head, g_begin + wave + WAVES * (i0 + lane), scales);
  };
  struct Group {
    u32x4 k[2 * NC], v[ND];
    int n;             // its valid tokens
    uint32_t scales;
  };
  auto fetch = [&](int i, Group& x) __attribute__((always_inline)) {
    const uint32_t g = __builtin_amdgcn_readlane(at, i - base);
    x.scales = __builtin_amdgcn_readlane(scales, i - base);
    x.n = g == kNoGroup ? 0 : min(len - 32 * (g_begin + wave + WAVES * i), 32);
    // a group that is not there: the pool's first is loaded and not used
    const uint64_t off = (uint64_t)(g == kNoGroup ? 0u : g) * kGroup;
    const u32x4* kp = reinterpret_cast<const u32x4*>(w.k_pages + off) + lane;
    const u32x4* vp = reinterpret_cast<const u32x4*>(w.v_pages + off + fh * (HD * 16)) + fr;
#pragma unroll
    for (int c = 0; c < 2 * NC; ++c) x.k[c] = kp[64 * c];
#pragma unroll
    for (int d = 0; d < ND; ++d) x.v[d] = vp[32 * d];
  };

  f32x16 oacc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) oacc[d] = f32x16{};
  float m = -INFINITY, l = 0.f;
  auto compute = [&](Group& x) __attribute__((always_inline)) {
    if (x.n == 0) return;
    f32x16 s{};
    const int ks = (int)x.scales;
    s = score_step<0, HD>(x.k[0], x.k[1], q, ks, s);
    if constexpr (NC == 2) s = score_step<1, HD>(x.k[2], x.k[3], q, ks, s);
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] *= w.scale_log2;
    if (x.n < 32) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (8 * (v >> 2) + 4 * fh + (v & 3) >= x.n) s[v] = -INFINITY;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) x.v[d][i] &= token_mask(i, fh, x.n);
    }
    float mx = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
    if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
      const float m_new = fmaxf(m, mx);
      const float a = __builtin_amdgcn_exp2f(m - m_new);   // the first group: 2^-inf = 0
      m = m_new;
      l *= a;
#pragma unroll
      for (int d = 0; d < ND; ++d) oacc[d] *= a;
    }
    bf16x8 p[2];
    float lp[2] = {0.f, 0.f};
#pragma unroll
    for (int v = 0; v < 16; v += 2) {
      const float p0 = __builtin_amdgcn_exp2f(s[v] - m), p1 = __builtin_amdgcn_exp2f(s[v + 1] - m);
      const bf16x2 pr = __builtin_convertvector((f32x2){p0, p1}, bf16x2);
      p[v >> 3][v & 7] = pr[0];
      p[v >> 3][(v & 7) + 1] = pr[1];
      lp[v >> 3] = add_pair(pr, lp[v >> 3]);
    }
    l += lp[0] + lp[1];
    const float vs = pow2(x.scales >> 8);
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8(x.v[d][0], x.v[d][1], vs), p[0], oacc[d], 0, 0, 0);
      oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8(x.v[d][2], x.v[d][3], vs), p[1], oacc[d], 0, 0, 0);
    }
  };

  for (int i0 = 0; i0 < n_mine; i0 += kWave) {
    look_up(i0);
    const int n = min(n_mine - i0, kWave);
    Group a, b;
    fetch(i0, a);
    for (int i = 0; i < n; i += 2) {
      if (i + 1 < n) fetch(i0 + i + 1, b);
      compute(a);
      if (i + 2 < n) fetch(i0 + i + 2, a);
      if (i + 1 < n) compute(b);
    }
  }
  l += __shfl_xor(l, 32, kWave);
  if (fh == 0) {
    part_m[wave][fr] = m;
    part_l[wave][fr] = l;
  }
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int v = 0; v < 16; ++v) part_o[wave][32 * d + 8 * (v >> 2) + 4 * fh + (v & 3)][fr] = oacc[d][v];
  __syncthreads();
  join_waves<HD, 32, WAVES>(part_o, part_m, part_l, 0, rows, it, w, O);
}

// ------------------------------------------------------------------- fp32

// 16 rows per workgroup; the waves share the groups of 32 tokens, each with an
// exact online softmax, on the fp32 matrix instruction: S^T = K Q^T on 16 keys
// leaves a lane four keys of one query, which feed O^T = V^T P^T from its
// registers.  A lane's four codes of an operand are one dword of the page,
// converted exactly.  Latency-bound at the small configuration's sizes.
template <int HD>
__global__ __launch_bounds__(256) void cached_attn_f32(const float* __restrict__ Q, float* __restrict__ O, CachedWork w) {
  constexpr int NB = HD / 16, kGroup = 32 * HD, WAVES = 4;
  __shared__ float part_o[WAVES][HD][17];
  __shared__ float part_m[WAVES][16], part_l[WAVES][16];
  Item it;
  if (!find_item(w, it)) return;
  const int req = w.req[it.i];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g4 = lane >> 4;
  const int rows = w.q_len[it.i] * w.group;
  const int row = min(it.tile * 16 + r, rows - 1);
  const float* qp = Q + (int64_t)(w.q_start[it.i] + row / w.group) * w.q_stride +
                    (it.head * w.group + row % w.group) * HD + 4 * g4;
  f32x4 q[NB], acc[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    q[c] = *reinterpret_cast<const f32x4*>(qp + 16 * c);
    acc[c] = f32x4{};
  }
  const int len = length_of(w, req);
  const int all = (len + 31) / 32;
  const int per = (all + w.pieces - 1) / w.pieces;
  const int g_begin = min(it.piece * per, all), g_end = min(g_begin + per, all);
  float m = -INFINITY, l = 0.f;
  for (int g = g_begin + wave; g < g_end; g += WAVES) {
    uint32_t scales;
    const uint32_t at = __builtin_amdgcn_readfirstlane(find_group(w, req, it.head, g, scales));
    if (at == kNoGroup) continue;
    const float ks = pow2(scales & 0xFF) * w.scale_log2, vs = pow2(scales >> 8);
    const char* kp = w.k_pages + (uint64_t)at * kGroup;
    const char* vp = w.v_pages + (uint64_t)at * kGroup;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int n = len - 32 * g - 16 * h;   // keys from here on
      if (n <= 0) break;
      uint32_t kw[NB], vw[NB];
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        kw[c] = *reinterpret_cast<const uint32_t*>(kp + c * 512 + (16 * h + r) * 16 + 4 * g4);
        // tokens 16 h + 4 g4 + 0 .. 3: slots 4 i + 0 .. 3 of f = g4 % 2, i = 2 h + g4 / 2
        vw[c] = *reinterpret_cast<const uint32_t*>(vp + (g4 & 1) * (HD * 16) + (16 * c + r) * 16 + 4 * (2 * h + (g4 >> 1)));
        if (n < 16) vw[c] &= token_mask(0, 0, n - 4 * g4);
      }
      f32x4 s{};
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)kw[c], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)kw[c], true);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(a[0], q[c][0], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(a[1], q[c][1], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(b[0], q[c][2], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(b[1], q[c][3], s, 0, 0, 0);
      }
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] = 4 * g4 + e < n ? s[e] * ks : -INFINITY;
        mx = fmaxf(mx, s[e]);
      }
      mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
      mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
      const float m_new = fmaxf(m, mx);
      const float ref = m_new == -INFINITY ? 0.f : m_new;   // scores of -inf only so far
      const float a = exp2f(m - ref);
      f32x4 p;
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = exp2f(s[e] - ref);
      l = l * a + ((p[0] + p[1]) + (p[2] + p[3]));
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8((int)vw[c], false) * vs;
        const f32x2 y = __builtin_amdgcn_cvt_pk_f32_fp8((int)vw[c], true) * vs;
        acc[c] *= a;
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[0], p[0], acc[c], 0, 0, 0);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[1], p[1], acc[c], 0, 0, 0);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[0], p[2], acc[c], 0, 0, 0);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[1], p[3], acc[c], 0, 0, 0);
      }
      m = m_new;
    }
  }
  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  if (g4 == 0) {
    part_m[wave][r] = m;
    part_l[wave][r] = l;
  }
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) part_o[wave][16 * c + 4 * g4 + e][r] = acc[c][e];
  __syncthreads();
  join_waves<HD, 16, WAVES>(part_o, part_m, part_l, it.tile * 16, rows, it, w, O);
}

// The key pieces of every row joined in order: O = sum_p 2^(m_p - m) O_p /
// sum_p 2^(m_p - m) l_p over the pieces that had keys, m their largest
// reference.  Four channels per thread.
template <int HD, typename T>
__global__ __launch_bounds__(256) void cached_attn_merge(T* __restrict__ O, int64_t o_stride, const float* __restrict__ part,
                                                         int pieces, int64_t rows, int n_heads) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t id = e / (HD / 4);
  const int d = (int)(e % (HD / 4)) * 4;
  if (id >= rows) return;
  const f32x2* ml = reinterpret_cast<const f32x2*>(part + pieces * rows * HD);
  float top = -INFINITY;
  for (int p = 0; p < pieces; ++p) {
    const f32x2 x = ml[p * rows + id];
    if (x[1] != 0.f) top = fmaxf(top, x[0]);
  }
  float l = 0.f;
  f32x4 o{};
  for (int p = 0; p < pieces; ++p) {
    const f32x2 x = ml[p * rows + id];
    if (x[1] == 0.f) continue;   // no keys
    const float a = exp2f(x[0] - top);
    l = fmaf(a, x[1], l);
    o += *reinterpret_cast<const f32x4*>(part + (p * rows + id) * HD + d) * a;
  }
  const float inv = l != 0.f ? 1.0f / l : 0.f;
  T* op = O + (id / n_heads) * o_stride + (id % n_heads) * HD + d;
#pragma unroll
  for (int j = 0; j < 4; ++j) op[j] = from_f<T>(o[j] * inv);
}

// ------------------------------------------------------------------ launch

enum Shape { kMany, kFew, kF32 };

struct CachedPlan {
  Shape shape;
  int tile_rows, pieces;
};

// Key pieces per item: enough workgroups for the compute units' slots, as long
// as a piece stays at least `min_unit` units of keys long.  The bound of the
// lengths stands for the lengths, which are device memory.
CachedPlan plan(const CachedAttnArgs& p, int cus) {
  CachedPlan pl;
  const int group = p.n_heads / p.n_kv_heads;
  int64_t most = 0;
  for (int r = 0; r < p.cq.n_req; ++r) most = std::max<int64_t>(most, (int64_t)(p.cq.cu[r + 1] - p.cq.cu[r]) * group);
  pl.shape = p.dtype == DIT_F32 ? kF32 : most <= 32 ? kFew : kMany;
  pl.tile_rows = pl.shape == kF32 ? 16 : pl.shape == kFew ? 32 : 128;
  int64_t items = 0;
  for (int r = 0; r < p.cq.n_req; ++r)
    items += ((int64_t)(p.cq.cu[r + 1] - p.cq.cu[r]) * group + pl.tile_rows - 1) / pl.tile_rows * p.n_kv_heads;
  pl.pieces = 1;
  if (items == 0) return pl;
  const int units = (p.max_len + 63) / 64;                 // tiles of 64 tokens
  const int64_t slots = 2 * (int64_t)cus;                  // workgroups that run at once
  const int min_units = pl.shape == kMany ? 8 : 16;        // 512 / 1024 tokens
  const int64_t most_pieces = std::min<int64_t>(64, units / min_units);
  if (pl.shape == kMany) {
    // rounds of workgroups x tiles per piece, and about 6 tiles' time per round for queries and output
    int64_t best = 0;
    for (int64_t s = 1; s <= std::max<int64_t>(1, most_pieces); ++s) {
      const int64_t cost = (items * s + slots - 1) / slots * ((units + s - 1) / s + 6 + (s > 1 ? 2 : 0));
      if (best == 0 || cost < best) {
        best = cost;
        pl.pieces = (int)s;
      }
    }
  } else {
    pl.pieces = (int)std::max<int64_t>(1, std::min<int64_t>(most_pieces, (2 * slots + items - 1) / items));
  }
  return pl;
}

int64_t part_floats(const CachedAttnArgs& p, int pieces) {
  return (int64_t)pieces * p.cq.cu[p.cq.n_req] * p.n_heads * (p.head_dim + 2);
}

}  // namespace

size_t cached_attention_ws(const CachedAttnArgs& p) {
  const CachedPlan pl = plan(p, cu_count());
  return pl.pieces > 1 ? (size_t)part_floats(p, pl.pieces) * 4 : 0;
}

hipError_t launch_cached_attention(const CachedAttnArgs& p, void* ws, hipStream_t s) {
  const CachedPlan pl = plan(p, cu_count());
  CachedWork w{};
  w.pieces = pl.pieces;
  w.n_pages = p.n_pages; w.page_shift = p.page_shift; w.max_pages = p.max_pages; w.max_len = p.max_len;
  w.n_heads = p.n_heads; w.n_kv_heads = p.n_kv_heads; w.group = p.n_heads / p.n_kv_heads;
  w.q_stride = p.q_stride; w.o_stride = p.o_stride;
  w.k_pages = p.k_pages; w.v_pages = p.v_pages; w.k_scale = p.k_scale; w.v_scale = p.v_scale;
  w.table = p.table; w.lens = p.lens;
  w.q_gain = (const bf16*)p.q_gain; w.q_eps = p.q_eps;
  w.scale_log2 = p.scale * 1.4426950408889634f;
  w.part = (float*)ws;
  w.part_rows = (int64_t)p.cq.cu[p.cq.n_req] * p.n_heads;
  int n = 0;
  int64_t items = 0;
  for (int r = 0; r < p.cq.n_req; ++r) {
    const int len = p.cq.cu[r + 1] - p.cq.cu[r];
    if (len == 0) continue;
    w.req[n] = r;
    w.q_start[n] = p.cq.cu[r];
    w.q_len[n] = len;
    w.tiles[n] = (int)(((int64_t)len * w.group + pl.tile_rows - 1) / pl.tile_rows);
    w.prefix[n] = (int)items;
    items += (int64_t)w.tiles[n] * p.n_kv_heads * pl.pieces;
    if (items > (1 << 23)) return hipErrorInvalidValue;   // a launch of fewer than 2^32 work-items
    w.prefix[++n] = (int)items;
  }
  w.n_req = n;
  if (items == 0) return hipSuccess;
  int per_xcd = 0;
  for (int x = 0; x < kXcds; ++x) {
    int64_t len = 0;
    for (int i = 0; i < n; ++i) {
      const int64_t k = w.prefix[i + 1] - w.prefix[i];
      len += (x + 1) * k / kXcds - x * k / kXcds;
    }
    per_xcd = std::max(per_xcd, (int)len);
  }
  const int grid = per_xcd * kXcds;
  auto merge = [&](auto tag, auto hd) {
    using T = decltype(tag);
    constexpr int HD = decltype(hd)::value;
    const int64_t threads = w.part_rows * (HD / 4);
    cached_attn_merge<HD, T><<<(unsigned)((threads + 255) / 256), 256, 0, s>>>((T*)p.o, p.o_stride, w.part, w.pieces,
                                                                            w.part_rows, p.n_heads);
  };
  auto run = [&](auto hd) {
    constexpr int HD = decltype(hd)::value;
    const bf16* q = (const bf16*)p.q;
    bf16* o = (bf16*)p.o;
    if (pl.shape == kF32) cached_attn_f32<HD><<<grid, 256, 0, s>>>((const float*)p.q, (float*)p.o, w);
    else if (pl.shape == kFew && p.q_gain) cached_attn_few<HD, true><<<grid, 256, 0, s>>>(q, o, w);
    else if (pl.shape == kFew) cached_attn_few<HD, false><<<grid, 256, 0, s>>>(q, o, w);
    else if (p.q_gain) cached_attn_many<HD, true><<<grid, 256, 0, s>>>(q, o, w);
    else cached_attn_many<HD, false><<<grid, 256, 0, s>>>(q, o, w);
    if (w.pieces > 1) {
      if (pl.shape == kF32) merge(float{}, hd);
      else merge(bf16{}, hd);
    }
  };
  if (p.head_dim == 64) run(std::integral_constant<int, 64>{});
  else run(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace dit
