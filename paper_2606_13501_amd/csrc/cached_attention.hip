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
// q = q1 + q2 exactly (values below 2^-13.8 of the largest of their 64 channels
// to 2^-21.8 of it), so two of the fp8 instructions, at twice the bf16 rate,
// give what a bf16 product of converted keys would, without the conversion.
// O^T = V^T P^T in bf16 MFMAs: v_cvt_scalef32_pk_bf16_fp8 turns two codes into
// bf16 with the page's scale, exactly.
//
// Softmax is fp32 in log2 units: a score is multiplied by scale * log2(e) in
// the multiply-add that takes off the row's reference.  (Multiplied into the
// query instead, it would have to be rounded to bf16 with it: the output was
// then 0.0037 off the exact one, root mean square, 0.0017 of which is its own
// rounding; now 0.0023.)  Probabilities are rounded to bf16, 8 significant bits
// each: the rest of the 0.0023.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace dit {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kXcds = 8;

// What the kernels need besides the caller's arguments: the row tiles of the
// requests that have queries.  An item is (request, key/value head, row tile),
// numbered with the row tiles of a head side by side.
struct CachedWork {
  int n_req;
  int shares;                       // 0: one workgroup per item; else see Share
  int unit_shift, min_share;        // log2 tokens of a unit; units
  int extra;                        // what an item costs beside its tokens, in units
  int tile_rows, merge_rows;
  int n_pages, page_shift, max_pages, max_len;
  int n_heads, n_kv_heads, group;   // group: query heads of a key/value head
  int64_t q_stride, o_stride;
  const char *k_pages, *v_pages;
  const uint8_t *k_scale, *v_scale;
  const int32_t *table, *lens;
  const bf16* q_gain;
  float q_eps, scale_log2;
  float* part;                      // shares > 0: fp32 [2 * shares][tile_rows][head_dim], then [..][tile_rows][2]
  int req[DIT_MAX_REQ];             // the request's index (its row of the table)
  int q_start[DIT_MAX_REQ];
  int q_len[DIT_MAX_REQ];
  int tiles[DIT_MAX_REQ];
  int prefix[DIT_MAX_REQ + 1];      // items before request i
};

// The request's cached length, within the table and the caller's bound.
__device__ __forceinline__ int length_of(const CachedWork& w, int r) { return min(max(w.lens[r], 0), w.max_len); }
__device__ __forceinline__ int units_of(const CachedWork& w, int len) { return (len + (1 << w.unit_shift) - 1) >> w.unit_shift; }

// What an item of the request costs, in units; one without tokens is left to
// cached_attn_merge.
__device__ __forceinline__ int cost_of(const CachedWork& w, int units) { return units > 0 ? units + w.extra : 0; }

// The requests' lengths, read once, and what their items cost; by the first wave,
// for the workgroup.  Nothing reads a length again: a length that is written
// meanwhile gives a wrong row, but no item outside its request.
struct Counted {
  int64_t ends[kWave];   // cost of requests 0 .. i
  int len[kWave];
};
__device__ __forceinline__ void count_units(const CachedWork& w, Counted& c) {
  if (threadIdx.x < kWave) {
    const int i = threadIdx.x;
    const int len = i < w.n_req ? length_of(w, w.req[i]) : 0;
    int64_t v = i < w.n_req ? (int64_t)w.tiles[i] * w.n_kv_heads * cost_of(w, units_of(w, len)) : 0;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int64_t below = __shfl_up(v, o, kWave);
      if (i >= o) v += below;
    }
    c.ends[i] = v;
    c.len[i] = len;
  }
  __syncthreads();
}
__device__ __forceinline__ int64_t share_of(const CachedWork& w, int64_t units) {
  return max((units + w.shares - 1) / w.shares, (int64_t)w.min_share);
}

// A value that is the same in every lane, as a scalar.
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// A workgroup's next piece of work: units u0 .. u1 of an item's tokens.
struct Segment {
  int i, head, tile;   // position in the work table, key/value head, row tile
  int len;             // the request's cached length
  int u0, u1;
  int slot;            // where its unfinished rows go (-1: it has all of the item's tokens)
};

// Where a row of the item's request lies: query row / group of its head row % group.
__device__ __forceinline__ int64_t query_at(const CachedWork& w, const Segment& g, int row, int64_t stride, int hd) {
  const int token = w.group == 1 ? row : row / w.group;   // (the division by a variable is 25 instructions)
  return (w.q_start[g.i] + token) * stride + (g.head * w.group + row - token * w.group) * hd;
}

// Workgroups are dispatched to the XCDs round-robin.
//
// shares == 0: each workgroup has one item, and each XCD the same contiguous
// eighth of every request's items: the row tiles that read the same keys stay
// on one XCD and share its L2.  The requests with the most tokens go first, so
// that short items fill the last round (only the device knows the lengths): five
// images on prompts of 18 to 512 tokens, 24 heads, 40.0 -> 38.9 us; where all
// lengths are equal the wait for them costs, 33.7 -> 34.3 us for four.
__device__ __forceinline__ bool whole_item(const CachedWork& w, Segment& g) {
  const int xcd = blockIdx.x % kXcds, at = blockIdx.x / kXcds;
  int item;
  g.i = 0;
  if (w.n_req == 1) {   // without waiting for a length
    g.len = length_of(w, w.req[0]);
    const int lo = xcd * w.prefix[1] / kXcds;   // (kMaxItems * 8 fits)
    item = lo + at;
    if (item >= (xcd + 1) * w.prefix[1] / kXcds) return false;
  } else {
    const int lane = threadIdx.x % kWave, i = min(lane, w.n_req - 1), len = length_of(w, w.req[i]);
    const int n = w.prefix[i + 1] - w.prefix[i];
    const int lo = xcd * n / kXcds, mine = (xcd + 1) * n / kXcds - lo;
    int start = 0;   // items of the requests before this lane's
    for (int j = 0; j < w.n_req; ++j) {
      const int lj = __builtin_amdgcn_readlane(len, j), nj = __builtin_amdgcn_readlane(mine, j);
      start += lj > len || (lj == len && j < i) ? nj : 0;
    }
    const uint64_t here = __builtin_amdgcn_ballot_w64(lane < w.n_req && at >= start && at < start + mine);
    if (here == 0) return false;
    g.i = __builtin_ctzll(here);
    item = __builtin_amdgcn_readlane(lo + at - start, g.i);
    g.len = __builtin_amdgcn_readlane(len, g.i);
  }
  g.head = item / w.tiles[g.i];
  g.tile = item - g.head * w.tiles[g.i];
  g.u0 = 0;
  g.len = __builtin_amdgcn_readfirstlane(g.len);
  g.u1 = units_of(w, g.len);
  g.slot = -1;
  return true;
}

// shares > 0: the costs of all items, in order, are dealt evenly to the
// workgroups, as many as run at once, so that all end together whatever the
// requests' lengths, which only the device knows.  An item's cost is its units
// and, before them, `extra` units for what every piece of work takes besides: a
// share of one long item is not behind one of many short ones.  An item that
// lies in several shares is joined by cached_attn_merge; a share has at most one
// item that began before it (slot 2 s) and one that ends after it (slot 2 s + 1).
// A share is worked off from its end: it begins with the item that ends after it,
// at that item's first token, so the workgroups that read one head's tokens,
// their shares about an item long, are at the same tokens at the same time, and
// one XCD's L2 serves them (from its beginning, each a little further on than
// the last, 1,560 x 31,200 tokens x 40 heads read 3.6 GB past the L2 and took
// 912 us; now 0.39 GB and 856 us).
struct Share {
  int s;
  int64_t pos, end;
};
__device__ __forceinline__ Share my_share(const CachedWork& w, Counted& c) {
  count_units(w, c);
  const int64_t all = uniform(c.ends[kWave - 1]), share = uniform(share_of(w, all));
  Share x;
  x.s = (blockIdx.x % kXcds) * (w.shares / kXcds) + blockIdx.x / kXcds;
  x.pos = x.s * share;
  x.end = min(x.pos + share, all);
  return x;
}
__device__ __forceinline__ bool next_segment(const CachedWork& w, const Counted& c, Share& x, Segment& g) {
  while (x.pos < x.end) {
    int64_t start = 0, upto = uniform(c.ends[0]);
    int r = 0;
    while (upto < x.end) {
      start = upto;
      upto = uniform(c.ends[++r]);
    }
    g.len = __builtin_amdgcn_readfirstlane(c.len[r]);
    const int units = units_of(w, g.len);
    const int cost = cost_of(w, units);
    const int64_t item = uniform((x.end - 1 - start) / cost);
    const int64_t begin = start + item * cost;
    const int from = (int)max(x.pos - begin, (int64_t)0), to = (int)(x.end - begin);
    x.end = begin + from;
    g.u0 = max(from - w.extra, 0);
    g.u1 = max(to - w.extra, 0);
    if (g.u1 == g.u0) continue;
    g.i = r;
    g.head = __builtin_amdgcn_readfirstlane((int)(item / w.tiles[r]));
    g.tile = (int)(item - (int64_t)g.head * w.tiles[r]);
    g.slot = g.u1 - g.u0 == units ? -1 : 2 * x.s + (g.u0 == 0);
    return true;
  }
  return false;
}

// Position of a group of 32 tokens in the pool, in groups (its page, head and
// place in the page), and its two scale bytes; none where `is` is false or the
// table names no page of the pool.  Without branches, and reading the table and
// the scales in any case (at entries that exist): nothing waits for the length,
// nor the tokens' loads for the scales.
constexpr uint32_t kNoGroup = 0xFFFFFFFFu;
struct GroupAt {
  uint32_t at;
  uint8_t k_scale, v_scale;
  __device__ __forceinline__ uint32_t scales() const { return at == kNoGroup ? 0x7F7Fu : k_scale | (uint32_t)v_scale << 8; }
};
__device__ __forceinline__ GroupAt find_group(const CachedWork& w, int r, int head, int g, bool is) {
  const int gs = w.page_shift - 5;   // log2 groups per page
  const int page = w.table[(int64_t)r * w.max_pages + min(g >> gs, w.max_pages - 1)];
  is &= (uint32_t)page < (uint32_t)w.n_pages;
  const uint32_t slot = (is ? (uint32_t)page : 0u) * w.n_kv_heads + head;
  return {is ? (slot << gs) + (g & ((1 << gs) - 1)) : kNoGroup, w.k_scale[slot], w.v_scale[slot]};
}

// Sum and maximum of a lane's value and that of the lane 32 (or 16) apart.
template <int N> __device__ __forceinline__ u32x2 swap_lanes(uint32_t x) {
  if constexpr (N == 32) {
    const auto sw = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return u32x2{sw[0], sw[1]};
  } else {
    const auto sw = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return u32x2{sw[0], sw[1]};
  }
}
template <int N> __device__ __forceinline__ float pair_max(float x) {
  const u32x2 sw = swap_lanes<N>(__float_as_uint(x));
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
template <int N> __device__ __forceinline__ float pair_sum(float x) {
  const u32x2 sw = swap_lanes<N>(__float_as_uint(x));
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

__device__ __forceinline__ float pow2(uint32_t biased) { return __uint_as_float(biased << 23); }

// This lane's query row as the B operand of S^T: channels 64 c + 32 h + 16 f
// .. +15 of the row (f: the lane's half; h: 0, 1), with QNORM RMS-normalised and
// rounded to bf16, split into two e4m3 parts with one power of two per row and
// 64 channels (the same byte in both lanes of a row: the instruction's blocks
// of 32 channels each span both).
template <int HD> struct QFrag {
  i32x8 hi[HD / 64], lo[HD / 64];
  int scales;   // byte 2 c: of hi[c], byte 2 c + 1: of lo[c] (smaller by 2^-4)
};

template <int HD>
__device__ __forceinline__ void load_row(const bf16* row, int f, bf16x8 (&raw)[HD / 16]) {
#pragma unroll
  for (int i = 0; i < HD / 16; ++i)
    raw[i] = *reinterpret_cast<const bf16x8*>(row + 32 * (i / 2) + 16 * f + 8 * (i % 2));
}

template <int HD, bool QNORM>
__device__ __forceinline__ void split_row(const bf16x8 (&raw)[HD / 16], int f, const CachedWork& w, QFrag<HD>& q) {
  constexpr int NC = HD / 64;
  float mul = 1.f;
  bf16x8 gain[QNORM ? 4 * NC : 1];
  if constexpr (QNORM) {
    // RMSNorm over the head: this lane holds half of its values, the lane 32 apart the other half
    load_row<HD>(w.q_gain, f, gain);
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * NC; ++i) {
      const f32x8 x = __builtin_convertvector(raw[i], f32x8);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
    }
    ss = pair_sum<32>(ss);
    mul = rsqrtf(ss * (1.0f / HD) + w.q_eps);
  }
  uint32_t bytes = 0;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    bf16x8 x[4];
    uint32_t top = 0;   // the largest magnitude, as fp32 bits
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = raw[4 * c + i];
      if constexpr (QNORM)
        x[i] = __builtin_convertvector(__builtin_convertvector(x[i], f32x8) * mul *
                                           __builtin_convertvector(gain[4 * c + i], f32x8), bf16x8);
      const u32x4 bits = __builtin_bit_cast(u32x4, x[i]);
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max(top, max(bits[e] << 16 & 0x7FFF0000u, bits[e] & 0x7FFF0000u));
    }
    const u32x2 both = swap_lanes<32>(top);
    top = max(both[0], both[1]);
    // smallest power of two with every value of the row's 64 channels (this
    // lane's and the lane's 32 apart) at most 448 = 1.75 * 2^8 of it; 16 and more,
    // so that the low part's byte stays positive.  A row with an infinity or NaN
    // gets the scale NaN, and with it its output.
    const uint32_t s = (uint32_t)max((int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u), 16);
    bytes |= (top >= 0x7F800000u ? 0xFFFFu : s | (s - 4) << 8) << (16 * c);
    const float hi_scale = pow2(s), lo_scale = pow2(s - 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bf16x2 x0 = {x[i / 2][4 * (i % 2)], x[i / 2][4 * (i % 2) + 1]};
      const bf16x2 x1 = {x[i / 2][4 * (i % 2) + 2], x[i / 2][4 * (i % 2) + 3]};
      i16x2 hw = {0, 0}, lw = {0, 0};
      hw = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hw, x0, hi_scale, false);
      hw = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hw, x1, hi_scale, true);
      const int h = __builtin_bit_cast(int, hw);
      const f32x2 h0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(h, hi_scale, false);
      const f32x2 h1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(h, hi_scale, true);
      lw = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lw, (float)x0[0] - h0[0], (float)x0[1] - h0[1], lo_scale, false);
      lw = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lw, (float)x1[0] - h1[0], (float)x1[1] - h1[1], lo_scale, true);
      q.hi[c][i] = h;
      q.lo[c][i] = __builtin_bit_cast(int, lw);
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

// the same for two groups of keys
template <int C, int HD>
__device__ __forceinline__ void score_step(const u32x4& a0, const u32x4& a1, const u32x4& b0, const u32x4& b1,
                                           const QFrag<HD>& q, const int (&ks)[2], f32x16 (&acc)[2]) {
  const i32x8 a = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
  const i32x8 b = {(int)b0[0], (int)b0[1], (int)b0[2], (int)b0[3], (int)b1[0], (int)b1[1], (int)b1[2], (int)b1[3]};
  acc[0] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q.hi[C], acc[0], 0, 0, 0, ks[0], 2 * C, q.scales);
  acc[1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, q.hi[C], acc[1], 0, 0, 0, ks[1], 2 * C, q.scales);
  acc[0] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q.lo[C], acc[0], 0, 0, 0, ks[0], 2 * C + 1, q.scales);
  acc[1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, q.lo[C], acc[1], 0, 0, 0, ks[1], 2 * C + 1, q.scales);
}

// 8 codes (two dwords) of one value channel -> bf16 with the page's scale
__device__ __forceinline__ bf16x8 values8(uint32_t w0, uint32_t w1, float vs) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, vs, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, vs, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, vs, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, vs, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
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

constexpr float kHeadroom = 18446744073709551616.0f;   // 2^64, bound of a row sum
constexpr float kFarScore = 4096.f;                    // bound of a row's reference
constexpr uint32_t kLargeScale = 127 + 48;             // bound of a value's scale byte: 2^64 * 448 * 2^48 is below 2^121

// 4 waves of 32 rows, two workgroups per compute unit; tiles of 64 tokens (8 KB
// of keys and 8 KB of values at 128 channels: half of bf16) in an LDS ring of 4,
// asked for three and more tiles ahead.
//
// The row reference of the softmax is the first tile's row maximum for the
// whole pass, so the loop neither searches maxima nor rescales the output.
// The exponent is one multiply-add on the unrounded product, against a reference
// that is rounded: all probabilities of a row carry the same factor 2^e, e at most
// half a step of the reference.  Where that could matter (references past 2^12,
// from where the parts of a row no longer agree to 2^-13), a row's sum passes 2^64
// or values are so large that a product with a probability of 2^64 could pass
// fp32, the workgroup finds the maxima of the rounded products and runs again on
// these, the largest probability exactly 1.
//
// Bound by the matrix instructions at the clock that the power limit leaves:
// 2,048 queries x 31,200 tokens x 32 heads of 128 take 832 us, 1.26 PFLOP/s.
// (Before a head's workgroups read the same tokens together, 907 us, the matrix
// cores were busy for 68% of the cycles at 1.80 GHz.  Other orders of the same
// instructions reached 74% at 1.74 GHz, the next tile's score products dealt
// among this one's softmax, or 50% at 2.0 GHz, 64 rows per wave and one
// workgroup per compute unit, and took as long or longer.)  Short prompts: the
// first tokens and rows are waited for most of half the time; 32,760 queries x
// 512 tokens x 40 heads of 128 take 388 us, 0.89 PFLOP/s and 1.7 TB/s (and 414 on
// a card that held 1.89 GHz meanwhile; five images on 18 to 512 tokens ran at 2.17).
template <int HD, bool QNORM, bool SHARES>
__global__ __launch_bounds__(256, 2) void cached_attn_many(const bf16* __restrict__ Q, bf16* __restrict__ O,
                                                           CachedWork w) {
  constexpr int NC = HD / 64;          // matrix instructions over the channels
  constexpr int ND = HD / 32;          // 32-channel blocks of the output
  constexpr int kGroup = 32 * HD;      // bytes of a group's keys
  constexpr int kSlot = 4 * kGroup;    // a tile: keys of both groups, then values of both
  constexpr int kLoads = kSlot / 4096; // 1 KB loads per wave and tile
  constexpr int kRing = 4;
  __shared__ __attribute__((aligned(1024))) char smem[kRing * kSlot];
  __shared__ int s_redo;
  __shared__ std::conditional_t<SHARES, Counted, int> counted;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fr = lane & 31, fh = lane >> 5;
  Segment it;
  Share share{};
  auto more = [&]() __attribute__((always_inline)) {
    if constexpr (SHARES) return next_segment(w, counted, share, it);
    else return false;
  };
  if constexpr (SHARES) {
    share = my_share(w, counted);
    if (!more()) return;
  } else {
    if (!whole_item(w, it)) return;
  }
  do {
    const int r = w.req[it.i];
    const int rows = w.q_len[it.i] * w.group;
    const int row0 = it.tile * 128 + wave * 32;   // this wave's rows: row0 ..
    const int len = it.len;
    const int t_begin = it.u0, t_end = it.u1;   // tiles: units of 64 tokens

    const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_char*)smem;
    const uint32_t voff = (uint32_t)(wave * 1024 % kGroup + lane * 16);
    // Where the next 64 tiles lie, one per lane: tile chunk0 + i's groups and
    // their scale bytes (keys, values, keys, values).
    int chunk0 = 0;
    uint32_t at0 = kNoGroup, at1 = kNoGroup, scales = 0;
    auto issue = [&](int t) __attribute__((always_inline)) {
      const uint32_t lds = lds_base + (uint32_t)((t % kRing) * kSlot + wave * 1024);
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int part = (wave + 4 * u) * 1024 / kGroup;   // 0, 1: keys of the groups; 2, 3: values
        const uint32_t g = __builtin_amdgcn_readlane(part & 1 ? at1 : at0, t - chunk0);
        const uint64_t pool = (uint64_t)(uintptr_t)(part >> 1 ? w.v_pages : w.k_pages);
        const uint64_t base = pool + (uint64_t)(g == kNoGroup ? 0u : g) * kGroup;
        const u32x4 desc = {(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, g == kNoGroup ? 0u : (uint32_t)kGroup,
                            0x00020000u};
        if (u == 0) load_lds16<0>(desc, voff, lds);
        else if (u == 1) load_lds16<4096>(desc, voff, lds);
        else if (u == 2) load_lds16<8192>(desc, voff, lds);
        else load_lds16<12288>(desc, voff, lds);
      }
    };

    // tiles c0 .. c1 - 1 (at most 64) are next: the first ones on their way, after
    // what `before` asks for (behind the lookup, which would wait for it)
    bool any_bad = false;   // some group before the request's end is missing
    auto begin_chunk = [&](int c0, int c1, auto before) __attribute__((always_inline)) {
      chunk0 = c0;
      const int t = c0 + lane;
      const bool is0 = t < c1, is1 = is0 && 64 * t + 32 < len;
      const GroupAt a = find_group(w, r, it.head, 2 * t, is0), b = find_group(w, r, it.head, 2 * t + 1, is1);
      at0 = a.at;
      at1 = b.at;
      any_bad = __builtin_amdgcn_ballot_w64((is0 && at0 == kNoGroup) || (is1 && at1 == kNoGroup)) != 0;
      __syncthreads();   // the tiles before have been read
      before();
      const int n = min(4, c1 - c0);
      for (int t = 0; t < n; ++t) issue(c0 + t);
      scales = a.scales() | b.scales() << 16;
    };
    bf16x8 raw[HD / 16];
    begin_chunk(t_begin, min(t_begin + kWave, t_end), [&]() __attribute__((always_inline)) {
      load_row<HD>(Q + query_at(w, it, min(row0 + fr, rows - 1), w.q_stride, HD), fh, raw);
    });
    bool begun = true;
    QFrag<HD> q;
    split_row<HD, QNORM>(raw, fh, w, q);
    f32x16 oacc[ND];
    float l_run[2], m_ref = 0.f, x_max = -INFINITY;
    bool large = false;   // some page of the tokens has values past kLargeScale
    // what a tile is for: the reference, the first pass against it, the maxima of
    // the rounded products, the last pass against those
    enum { kFirst, kAgainstFirst, kFindMax, kAgainstMax } phase = kFirst;
    const float c = w.scale_log2;
    const float off_score = c < 0.f ? INFINITY : -INFINITY;   // times c: -inf

    // S of tile t: all key pieces first, then the products of both halves in
    // turn: each has the time of the other to come out before it goes on
    auto scores = [&](int t, f32x16 (&s)[2]) __attribute__((always_inline)) {
      const char* slot = smem + (t % kRing) * kSlot;
      const uint32_t sc = __builtin_amdgcn_readlane(scales, t - chunk0);
      const int ks[2] = {(int)sc, (int)(sc >> 16)};
      u32x4 kf[2][2 * NC];
#pragma unroll
      for (int i = 0; i < 2 * NC; ++i)
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) kf[hb][i] = reinterpret_cast<const u32x4*>(slot + hb * kGroup)[64 * i + lane];
      s[0] = s[1] = f32x16{};
      score_step<0, HD>(kf[0][0], kf[0][1], kf[1][0], kf[1][1], q, ks, s);
      if constexpr (NC == 2) score_step<1, HD>(kf[0][2], kf[0][3], kf[1][2], kf[1][3], q, ks, s);
    };
    // P of the scores (times c: log2 units), and O += V P
    auto output = [&](int t, const f32x16 (&s)[2], float c) __attribute__((always_inline)) {
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
          l_run[0] += p0;
          l_run[1] += p1;
        }
      const char* slot = smem + (t % kRing) * kSlot;
      const uint32_t sc = __builtin_amdgcn_readlane(scales, t - chunk0);
#pragma unroll
      for (int hb = 0; hb < 2; ++hb) {
        const float vs = pow2(hb ? sc >> 24 : (sc >> 8) & 0xFFu);
        const u32x4* vp = reinterpret_cast<const u32x4*>(slot + (2 + hb) * kGroup + fh * (HD * 16)) + fr;
#pragma unroll
        for (int db = 0; db < ND; ++db) {
          const u32x4 x = vp[32 * db];
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8(x[0], x[1], vs), p[2 * hb], oacc[db], 0, 0, 0);
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8(x[2], x[3], vs), p[2 * hb + 1], oacc[db], 0, 0, 0);
        }
      }
    };

    auto run_pass = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int db = 0; db < ND; ++db) oacc[db] = f32x16{};
      l_run[0] = l_run[1] = 0.f;
      for (int c0 = t_begin; c0 < t_end; c0 += kWave) {
        const int c1 = min(c0 + kWave, t_end);
        if (!begun) begin_chunk(c0, c1, [] {});
        begun = false;
        wait_vmcnt<0>();   // the first tiles, asked for with the queries and scales; only tile loads are counted from here on
        __syncthreads();
        large |= __builtin_amdgcn_ballot_w64((scales >> 8 & 0xFFu) > kLargeScale || scales >> 24 > kLargeScale) != 0;
        // tile t is done: tile t + 1 in LDS for every wave; tile t + 4 into the slot of t
        auto advance = [&](int t) __attribute__((always_inline)) {
          if (t + 1 >= c1) return;
          if (t + 3 < c1) wait_vmcnt<2 * kLoads>();
          else if (t + 2 < c1) wait_vmcnt<kLoads>();
          else wait_vmcnt<0>();
          __syncthreads();
          if (t + 4 < c1) issue(t + 4);
        };
        for (int t = c0; t < c1;) {
          if (!any_bad && phase == kAgainstFirst) {
            const int t_full = min(c1, len / 64);   // whole tiles
            for (; t < t_full; ++t) {
              // The older of two waves goes first wherever both could; with turns at a higher
              // priority the compute unit's two workgroups end more nearly together (849 ->
              // 833 us at the size above; with whole items it made no difference)
              if constexpr (SHARES) {
                if ((t ^ (blockIdx.x >> 8)) & 1) __builtin_amdgcn_s_setprio(1);
                else __builtin_amdgcn_s_setprio(0);
              }
              if (row0 < rows) {
                f32x16 s[2];
                scores(t, s);
                output(t, s, c);
              }
              advance(t);
            }
            if (t >= c1) break;
          }
          {
            const bool masked = any_bad || 64 * (t + 1) > len;
            int n0 = 32, n1 = 32;
            f32x16 s[2];
            scores(t, s);
            if (masked) {
              // it ends early or lacks a page: the scores of tokens that do not count
              // become -inf, and the workgroup clears their value codes (whatever the
              // page held before, NaN among them, which a probability of 0 would not
              // take out of the product)
              n0 = __builtin_amdgcn_readlane(at0, t - chunk0) == kNoGroup ? 0 : min(max(len - 64 * t, 0), 32);
              n1 = __builtin_amdgcn_readlane(at1, t - chunk0) == kNoGroup ? 0 : min(max(len - 64 * t - 32, 0), 32);
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
#pragma unroll
              for (int hb = 0; hb < 2; ++hb)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                  if (8 * (v >> 2) + 4 * fh + (v & 3) >= (hb ? n1 : n0)) s[hb][v] = off_score;
            }
            if (n0 + n1 > 0) {   // (nothing there: the reference waits for the next tile)
              const float unit = phase >= kFindMax ? 1.f : c;
              if (phase >= kFindMax) {
                s[0] *= c;
                s[1] *= c;
              }
              if (phase == kFirst || phase == kFindMax) {
                float mx = -INFINITY;
#pragma unroll
                for (int v = 0; v < 16; ++v) mx = fmaxf(mx, fmaxf(s[0][v] * unit, s[1][v] * unit));
                if (phase == kFindMax) x_max = fmaxf(x_max, mx);
                else m_ref = pair_max<32>(mx);
              }
              if (phase == kFirst) phase = kAgainstFirst;
              if (phase != kFindMax) output(t, s, unit);
            }
          }
          advance(t);
          ++t;
        }
      }
    };

    float l_tot;
#pragma unroll 1
    for (;;) {
      run_pass();
      if (phase == kFindMax) {
        m_ref = pair_max<32>(x_max);
        if (m_ref == -INFINITY) m_ref = 0.f;   // scores of -inf only: probabilities of 0
        phase = kAgainstMax;
        continue;
      }
      l_tot = pair_sum<32>(l_run[0] + l_run[1]);
      if (tid == 0) s_redo = 0;
      __syncthreads();   // (and every wave has read its last tile: the ring is free)
      if (phase == kAgainstMax) break;
      const bool fine = l_tot <= kHeadroom && fabsf(m_ref) <= kFarScore && !large;
      if (__builtin_amdgcn_ballot_w64(!fine) != 0 && lane == 0) s_redo = 1;
      __syncthreads();
      if (__builtin_amdgcn_readfirstlane(s_redo) == 0) break;
      phase = kFindMax;
    }

    // oacc[db][4 i + j]: channel 32 db + 8 i + 4 fh + j of the lane's row
    if (it.slot >= 0) {
      if (row0 + fr >= rows) continue;
      const int64_t at = (int64_t)it.slot * 128 + wave * 32 + fr;
      float* po = w.part + at * HD + 4 * fh;
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(po + 32 * db + 8 * i) =
              f32x4{oacc[db][4 * i], oacc[db][4 * i + 1], oacc[db][4 * i + 2], oacc[db][4 * i + 3]};
      if (fh == 0) *reinterpret_cast<f32x2*>(w.part + (int64_t)2 * w.shares * 128 * HD + 2 * at) = f32x2{m_ref, l_tot};
      continue;
    }
    // whole rows: through this wave's part of the ring, so that they are stored 16
    // bytes per lane and whole rows at a time (chunk i of row n lies at i ^ n % 16)
    char* stage = smem + wave * 32 * HD * 2;
    constexpr int kChunks = HD / 8;              // 16-byte chunks of a row
    const float inv = l_tot != 0.f ? 1.0f / l_tot : 0.f;   // no keys: a row of zeros
#pragma unroll
    for (int db = 0; db < ND; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bf16x4 ov;
#pragma unroll
        for (int j = 0; j < 4; ++j) ov[j] = (bf16)(oacc[db][4 * i + j] * inv);
        *reinterpret_cast<bf16x4*>(stage + fr * (HD * 2) + (((4 * db + i) ^ (fr % kChunks)) * 16) + 8 * fh) = ov;
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 32 * kChunks / 64; ++k) {
      const int n = (k * 64 + lane) / kChunks, i = lane % kChunks;
      const u32x4 x = *reinterpret_cast<const u32x4*>(stage + n * (HD * 2) + ((i ^ (n % kChunks)) * 16));
      const int row = row0 + n;
      if (row < rows)
        *reinterpret_cast<u32x4*>(O + query_at(w, it, row, w.o_stride, HD) + 8 * i) = x;
    }
    __builtin_amdgcn_wave_barrier();
  } while (more());
}

// ------------------------------------------------ the waves' shares, joined

// Row `row` of a workgroup's tile: WAVES partial outputs o[wave][row][channel],
// references m and sums l (log2 units; l 0: no keys), joined in wave order, then
// written to the output or, unfinished, to the segment's slot.  Four channels per
// thread (with one, 32 rows x 512 tokens x 40 heads took 18.6 us, now 11.6).
template <int HD, int ROWS, int WAVES, typename T>
__device__ __forceinline__ void join_waves(const float (&o)[WAVES][ROWS][HD + 4], const float (&m)[WAVES][ROWS],
                                           const float (&l)[WAVES][ROWS], int row0, int rows, const Segment& it,
                                           const CachedWork& w, T* O) {
  for (int e = threadIdx.x; e < min(ROWS, rows - row0) * (HD / 4); e += WAVES * kWave) {
    const int i = e / (HD / 4), d = e % (HD / 4) * 4;
    const int row = row0 + i;
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < WAVES; ++v)
      if (l[v][i] != 0.f) top = fmaxf(top, m[v][i]);
    float sum = 0.f;
    f32x4 acc{};
#pragma unroll
    for (int v = 0; v < WAVES; ++v)
      if (l[v][i] != 0.f) {
        const float a = exp2f(m[v][i] - top);
        sum = fmaf(a, l[v][i], sum);
        acc += *reinterpret_cast<const f32x4*>(&o[v][i][d]) * a;
      }
    if (it.slot >= 0) {
      const int64_t at = (int64_t)it.slot * ROWS + i;
      *reinterpret_cast<f32x4*>(w.part + at * HD + d) = acc;
      if (d == 0) *reinterpret_cast<f32x2*>(w.part + (int64_t)2 * w.shares * ROWS * HD + 2 * at) = f32x2{top, sum};
    } else {
      T* op = O + query_at(w, it, row, w.o_stride, HD) + d;
#pragma unroll
      for (int j = 0; j < 4; ++j) op[j] = from_f<T>(sum != 0.f ? acc[j] / sum : 0.f);
    }
  }
}

// -------------------------------------------------- bf16, few rows of a head

constexpr int kKeyWaves = 8;   // waves of a workgroup whose waves share the tokens

// At most 32 rows per head: the cache is read once and bounds the time, so the
// waves share the tokens, not the rows.  Each wave takes every 8th group of 32
// tokens of its segment, straight from global memory into registers in the
// operands' order (whole KiB per load), two groups ahead, with an exact online
// softmax; the waves meet in LDS, the shares in cached_attn_merge.
//
// HBM-bound on long histories: 16 single queries x 2,767 .. 32,760 tokens, 40
// heads on 8, take 121 us, 5.2 TB/s.  Latency-bound on one prompt: 1 query x 512
// tokens x 40 heads 9.0 us (the kernel above: 12.4; at 32 rows 11.6 and 13.1).
template <int HD, bool QNORM, bool SHARES>
__global__ __launch_bounds__(64 * kKeyWaves) void cached_attn_few(const bf16* __restrict__ Q, bf16* __restrict__ O,
                                                                  CachedWork w) {
  constexpr int NC = HD / 64, ND = HD / 32, kGroup = 32 * HD, WAVES = kKeyWaves;
  __shared__ __attribute__((aligned(16))) float part_o[WAVES][32][HD + 4];
  __shared__ float part_m[WAVES][32], part_l[WAVES][32];
  __shared__ std::conditional_t<SHARES, Counted, int> counted;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fr = lane & 31, fh = lane >> 5;
  Segment it;
  Share share{};
  auto more = [&]() __attribute__((always_inline)) {
    if constexpr (SHARES) return next_segment(w, counted, share, it);
    else return false;
  };
  if constexpr (SHARES) {
    share = my_share(w, counted);
    if (!more()) return;
  } else {
    if (!whole_item(w, it)) return;
  }
  do {
    const int r = w.req[it.i];
    const int rows = w.q_len[it.i] * w.group;
    const int row = min(fr, rows - 1);
    const int len = it.len;
    const int g_begin = 4 * it.u0, g_end = min(4 * it.u1, (len + 31) / 32);   // units of 128 tokens
    const int n_mine = max(0, (g_end - g_begin - wave + WAVES - 1) / WAVES);   // groups g_begin + wave + WAVES i

    uint32_t at = kNoGroup, scales = 0;   // lane i: this wave's group base + i
    int base = 0;
    auto look_up = [&](int i0) __attribute__((always_inline)) {
      base = i0;
      const GroupAt x = find_group(w, r, it.head, g_begin + wave + WAVES * (i0 + lane), i0 + lane < n_mine);
      at = x.at;
      scales = x.scales();
    };
    struct Group {
      u32x4 k[2 * NC], v[ND];
    };
    auto fetch = [&](int i, Group& x) __attribute__((always_inline)) {
      const uint32_t g = __builtin_amdgcn_readlane(at, i - base);
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
    QFrag<HD> q;
    auto compute = [&](int i, Group& x) __attribute__((always_inline)) {
      const bool there = __builtin_amdgcn_readlane(at, i - base) != kNoGroup;
      const uint32_t sc = __builtin_amdgcn_readlane(scales, i - base);
      const int n = there ? min(len - 32 * (g_begin + wave + WAVES * i), 32) : 0;   // its valid tokens
      if (n == 0) return;
      f32x16 s{};
      const int ks = (int)sc;
      s = score_step<0, HD>(x.k[0], x.k[1], q, ks, s);
      if constexpr (NC == 2) s = score_step<1, HD>(x.k[2], x.k[3], q, ks, s);
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] *= w.scale_log2;
      if (n < 32) {
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (8 * (v >> 2) + 4 * fh + (v & 3) >= n) s[v] = -INFINITY;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) x.v[d][i] &= token_mask(i, fh, n);
      }
      float mx = s[0];
#pragma unroll
      for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
      mx = pair_max<32>(mx);
      if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
        const float m_new = fmaxf(m, mx);
        const float a = __builtin_amdgcn_exp2f(m - (m_new == -INFINITY ? 0.f : m_new));   // the first group: 2^-inf = 0
        m = m_new;
        l *= a;
#pragma unroll
        for (int d = 0; d < ND; ++d) oacc[d] *= a;
      }
      const float ref = m == -INFINITY ? 0.f : m;   // scores of -inf only so far
      bf16x8 p[2];
      float lp[2] = {0.f, 0.f};
#pragma unroll
      for (int v = 0; v < 16; v += 2) {
        const float p0 = __builtin_amdgcn_exp2f(s[v] - ref), p1 = __builtin_amdgcn_exp2f(s[v + 1] - ref);
        const bf16x2 pr = __builtin_convertvector((f32x2){p0, p1}, bf16x2);
        p[v >> 3][v & 7] = pr[0];
        p[v >> 3][(v & 7) + 1] = pr[1];
        lp[0] += p0;
        lp[1] += p1;
      }
      l += lp[0] + lp[1];
      const float vs = pow2(sc >> 8);
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8(x.v[d][0], x.v[d][1], vs), p[0], oacc[d], 0, 0, 0);
        oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values8(x.v[d][2], x.v[d][3], vs), p[1], oacc[d], 0, 0, 0);
      }
    };

    // the first tokens are on their way before the queries are split (and looked up
    // before the queries are asked for: loads come back in their order)
    Group a{};
    bf16x8 raw[HD / 16];
    look_up(0);
    load_row<HD>(Q + query_at(w, it, row, w.q_stride, HD), fh, raw);
    if (n_mine > 0) fetch(0, a);
    split_row<HD, QNORM>(raw, fh, w, q);
    for (int i0 = 0; i0 < n_mine; i0 += kWave) {
      if (i0 > 0) {
        look_up(i0);
        fetch(i0, a);
      }
      const int n = min(n_mine - i0, kWave);
#pragma unroll 1
      for (int i = 0; i < n; ++i) {   // one copy of its code: few tokens wait for the instructions
        Group b = a;
        if (i + 1 < n) fetch(i0 + i + 1, b);
        compute(i0 + i, a);
        a = b;
      }
    }
    l = pair_sum<32>(l);
    __syncthreads();   // the previous segment's rows have been read
    if (fh == 0) {
      part_m[wave][fr] = m;
      part_l[wave][fr] = l;
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(&part_o[wave][fr][32 * d + 8 * i + 4 * fh]) =
            f32x4{oacc[d][4 * i], oacc[d][4 * i + 1], oacc[d][4 * i + 2], oacc[d][4 * i + 3]};
    __syncthreads();
    join_waves<HD, 32, WAVES>(part_o, part_m, part_l, 0, rows, it, w, O);
  } while (more());
}

// ------------------------------------------------------------------- fp32

// 16 rows per workgroup; the waves share the tokens in tiles of 16 (wave v has
// every 8th), each with an exact online softmax, on the fp32 matrix instruction:
// S^T = K Q^T on 16 keys leaves a lane four keys of one query, which feed O^T =
// V^T P^T from its registers.  A lane's four codes of an operand are one dword
// of the page, converted exactly.  Latency-bound at the small configuration's
// sizes (64 queries x 77 tokens x 6 heads of 64: 7.5 us): the next tile is asked
// for before the last is computed.  With many items the fp32 matrix rate is what
// is left (400 x 512 tokens x 40 heads of 128: 59 us, 30 us of it in matrix
// instructions); two workgroups of whole items per compute unit, at the price of
// two spilled registers, took it there from 87 (in shares, whose kernel needs 148
// registers at 128 channels, one fits).
template <int HD, bool SHARES>
__global__ __launch_bounds__(64 * kKeyWaves, SHARES ? 2 : 4) void cached_attn_f32(const float* __restrict__ Q, float* __restrict__ O,
                                                                  CachedWork w) {
  constexpr int NB = HD / 16, kGroup = 32 * HD, WAVES = kKeyWaves;
  __shared__ __attribute__((aligned(16))) float part_o[WAVES][16][HD + 4];
  __shared__ float part_m[WAVES][16], part_l[WAVES][16];
  __shared__ std::conditional_t<SHARES, Counted, int> counted;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g4 = lane >> 4;
  Segment it;
  Share share{};
  auto more = [&]() __attribute__((always_inline)) {
    if constexpr (SHARES) return next_segment(w, counted, share, it);
    else return false;
  };
  if constexpr (SHARES) {
    share = my_share(w, counted);
    if (!more()) return;
  } else {
    if (!whole_item(w, it)) return;
  }
  do {
    const int req = w.req[it.i];
    const int rows = w.q_len[it.i] * w.group;
    const int row = min(it.tile * 16 + r, rows - 1);
    const int len = it.len;
    const int t_begin = 8 * it.u0, t_end = min(8 * it.u1, (len + 15) / 16);   // units of 128 tokens
    const int n_mine = max(0, (t_end - t_begin - wave + WAVES - 1) / WAVES);   // tiles t_begin + wave + WAVES i
    uint32_t at = kNoGroup, scales = 0;   // lane i: the group of this wave's tile base + i
    int base = 0;
    auto look_up = [&](int i0) __attribute__((always_inline)) {
      base = i0;
      const GroupAt x = find_group(w, req, it.head, (t_begin + wave + WAVES * (i0 + lane)) / 2, i0 + lane < n_mine);
      at = x.at;
      scales = x.scales();
    };
    look_up(0);   // before the queries, for which it would wait
    const float* qp = Q + query_at(w, it, row, w.q_stride, HD) + 4 * g4;
    f32x4 q[NB], acc[NB];
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      q[c] = *reinterpret_cast<const f32x4*>(qp + 16 * c);
      acc[c] = f32x4{};
    }
    struct Tile {
      uint32_t k[NB], v[NB];
    };
    auto fetch = [&](int i, Tile& x) __attribute__((always_inline)) {
      const uint32_t g = __builtin_amdgcn_readlane(at, i - base);
      const int h = (t_begin + wave + WAVES * i) & 1;   // half of the group
      // a group that is not there: the pool's first is loaded and not used
      const uint64_t off = (uint64_t)(g == kNoGroup ? 0u : g) * kGroup;
      const char* kp = w.k_pages + off + (16 * h + r) * 16 + 4 * g4;
      // tokens 16 h + 4 g4 + 0 .. 3: slots 4 i + 0 .. 3 of f = g4 % 2, i = 2 h + g4 / 2
      const char* vp = w.v_pages + off + (g4 & 1) * (HD * 16) + r * 16 + 4 * (2 * h + (g4 >> 1));
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        x.k[c] = *reinterpret_cast<const uint32_t*>(kp + c * 512);
        x.v[c] = *reinterpret_cast<const uint32_t*>(vp + c * 256);
      }
    };
    float m = -INFINITY, l = 0.f;
    auto compute = [&](int i, Tile& x) __attribute__((always_inline)) {
      if (__builtin_amdgcn_readlane(at, i - base) == kNoGroup) return;
      const uint32_t sc = __builtin_amdgcn_readlane(scales, i - base);
      const float ks = pow2(sc & 0xFF) * w.scale_log2, vs = pow2(sc >> 8);
      const int n = len - 16 * (t_begin + wave + WAVES * i);   // keys from here on
      f32x4 s0{}, s1{};   // two sums: each product has the time of the other's to come out
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x.k[c], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)x.k[c], true);
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(a[0], q[c][0], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(a[1], q[c][1], s1, 0, 0, 0);
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(b[0], q[c][2], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(b[1], q[c][3], s1, 0, 0, 0);
      }
      f32x4 s = s0 + s1;
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] = 4 * g4 + e < n ? s[e] * ks : -INFINITY;
        mx = fmaxf(mx, s[e]);
      }
      mx = pair_max<32>(pair_max<16>(mx));
      const float m_new = fmaxf(m, mx);
      const float ref = m_new == -INFINITY ? 0.f : m_new;   // scores of -inf only so far
      const float a = exp2f(m - ref);
      f32x4 p;
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = exp2f(s[e] - ref);
      l = l * a + ((p[0] + p[1]) + (p[2] + p[3]));
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const uint32_t v = n < 16 ? x.v[c] & token_mask(0, 0, n - 4 * g4) : x.v[c];
        const f32x2 y = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, false) * vs, z = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, true) * vs;
        acc[c] *= a;
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[0], p[0], acc[c], 0, 0, 0);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[1], p[1], acc[c], 0, 0, 0);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(z[0], p[2], acc[c], 0, 0, 0);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(z[1], p[3], acc[c], 0, 0, 0);
      }
      m = m_new;
    };
    for (int i0 = 0; i0 < n_mine; i0 += kWave) {
      if (i0 > 0) look_up(i0);
      const int n = min(n_mine - i0, kWave);
      Tile a;
      fetch(i0, a);
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        Tile b = a;
        if (i + 1 < n) fetch(i0 + i + 1, b);
        compute(i0 + i, a);
        a = b;
      }
    }
    l = pair_sum<32>(pair_sum<16>(l));
    __syncthreads();   // the previous segment's rows have been read
    if (g4 == 0) {
      part_m[wave][r] = m;
      part_l[wave][r] = l;
    }
#pragma unroll
    for (int c = 0; c < NB; ++c) *reinterpret_cast<f32x4*>(&part_o[wave][r][16 * c + 4 * g4]) = acc[c];
    __syncthreads();
    join_waves<HD, 16, WAVES>(part_o, part_m, part_l, it.tile * 16, rows, it, w, O);
  } while (more());
}

// The rows whose tokens lay in several shares, joined in the shares' order: O =
// sum_p 2^(m_p - m) O_p / sum_p 2^(m_p - m) l_p over the parts p that had keys,
// m their largest reference.  Rows without tokens are in no share and get zeros
// here.  A workgroup has up to 16 rows of one item, so that the search for its
// parts, with its divisions, is done once; four channels per thread and row.
// (With each thread searching for its row: 28 us for 62,400 rows of 2 parts, now
// 21.)  Where a row has many parts the thread groups of a workgroup share them
// (105 rows x 25,649 tokens x 6 heads, 50 parts: 57 -> 34 us with it and the
// even costs).
struct Joined {
  float top, l;
  f32x4 o;
};
__device__ __forceinline__ void join(Joined& x, float top, float l, f32x4 o) {
  if (l == 0.f) return;   // no keys there
  const float m = fmaxf(x.top, top);
  const float a = exp2f(x.top - m), b = exp2f(top - m);   // (the first: 2^-inf = 0)
  x.l = fmaf(b, l, x.l * a);
  x.o = x.o * a + o * b;
  x.top = m;
}
template <int HD, typename T>
__global__ __launch_bounds__(256) void cached_attn_merge(T* __restrict__ O, CachedWork w) {
  constexpr int LANES = HD / 4, GROUPS = 256 / LANES;   // lanes of a row, rows at a time
  __shared__ Counted counted;
  __shared__ Joined halves[GROUPS][LANES];
  count_units(w, counted);
  const int per_item = w.tile_rows / w.merge_rows;
  const int item = blockIdx.x / per_item, at0 = blockIdx.x % per_item * w.merge_rows;
  const int lane = threadIdx.x % kWave, group = threadIdx.x / LANES, d = threadIdx.x % LANES * 4;
  Segment it;
  it.i = (int)__popcll(__builtin_amdgcn_ballot_w64(lane < w.n_req && w.prefix[min(lane, w.n_req - 1) + 1] <= item));
  const int nth = item - w.prefix[it.i];
  it.head = nth / w.tiles[it.i];
  it.tile = nth - it.head * w.tiles[it.i];
  const int units = __builtin_amdgcn_readfirstlane(units_of(w, counted.len[it.i]));
  int s0 = 0, s1 = -1;
  if (units > 0) {
    const int64_t first = uniform((it.i > 0 ? counted.ends[it.i - 1] : 0) + (int64_t)nth * cost_of(w, units) + w.extra);
    const int64_t share = uniform(share_of(w, counted.ends[kWave - 1]));
    s0 = (int)(first / share);
    s1 = (int)((first + units - 1) / share);
    if (s0 == s1) return;   // written by its workgroup
  }
  const f32x2* ml = reinterpret_cast<const f32x2*>(w.part + (int64_t)2 * w.shares * w.tile_rows * HD);
  // parts a .. b of row `at` of the tile, four parts' loads at a time, joined in order
  auto parts = [&](int at, int a, int b) __attribute__((always_inline)) {
    Joined y = {-INFINITY, 0.f, f32x4{}};
    for (int s = a; s <= b; s += 4) {
      f32x2 x[4];
      f32x4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int at_s = min(s + k, b);
        const int64_t slot_row = (int64_t)(2 * at_s + (at_s == s0)) * w.tile_rows + at;
        x[k] = ml[slot_row];
        v[k] = *reinterpret_cast<const f32x4*>(w.part + slot_row * HD + d);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (s + k <= b) join(y, x[k][0], x[k][1], v[k]);
    }
    return y;
  };
  auto write = [&](int row, const Joined& y) __attribute__((always_inline)) {
    const f32x4 o = y.o * (y.l != 0.f ? 1.0f / y.l : 0.f);
    T* op = O + query_at(w, it, row, w.o_stride, HD) + d;
#pragma unroll
    for (int j = 0; j < 4; ++j) op[j] = from_f<T>(o[j]);
  };
  const int row0 = it.tile * w.tile_rows;
  const int n = min(at0 + w.merge_rows, w.q_len[it.i] * w.group - row0);   // rows at0 .. n - 1 of the tile
  if (w.merge_rows >= GROUPS) {
    for (int at = at0 + group; at < n; at += GROUPS) write(row0 + at, parts(at, s0, s1));
  } else {
    const int per_row = GROUPS / w.merge_rows, at = at0 + group / per_row, g0 = group % per_row;
    const int each = (s1 - s0 + per_row) / per_row, a = s0 + g0 * each;
    if (at < n) halves[group][d / 4] = parts(at, a, min(a + each - 1, s1));
    __syncthreads();
    if (at < n && g0 == 0) {
      Joined y = halves[group][d / 4];
      for (int g = 1; g < per_row; ++g) join(y, halves[group + g][d / 4].top, halves[group + g][d / 4].l, halves[group + g][d / 4].o);
      write(row0 + at, y);
    }
  }
}

// ------------------------------------------------------------------ launch

constexpr int64_t kMaxItems = (1 << 22);   // 512 threads each: a launch of fewer than 2^32 work-items

enum Shape { kMany, kFew, kF32 };

struct CachedPlan {
  Shape shape;
  int tile_rows, unit_shift, min_share, extra, shares, merge_rows;
};

// The kernel, and whether its workgroups take whole items or even shares of all
// tokens: whichever an estimate from measured times finds shorter.  Shares cost
// a write, a read and a kernel of joining; whole items leave compute units idle
// in the last round.  Measured, shares / whole: 1,560 rows x 31,200 tokens x 40
// heads 846 / 1,153 us, 256 x 8,192 x 40 61 / 128, 3,000 x 1,500 x 40 117 / 96,
// 700 x 1,500 x 24 40 / 31, single queries on 4,000 tokens x 40 18.6 / 23.8, on
// 1,200 14.2 / 12.4.  (Within 5% of each other the estimate may miss: 6,000 x
// 6,000 x 40 654 / 634.)  The bound of the lengths stands for the lengths, which
// are device memory.  The costs are those of 128 channels, and of one workgroup
// per compute unit in fp32; they stand for 64 channels, and for whole fp32 items,
// of which two run, as well.
//
// A share has at least 256 tokens (with 512, 42 rows x 3,628 tokens x 6 heads
// took 20 us, now 16).  An item's cost beside its tokens, the latencies of
// finding and loading its first ones and of writing its part (9 us where a tile
// of 64 takes 1), is counted as 512 tokens, 1,536 where the waves share the
// tokens: 13 requests of 3 to 31,478 tokens, 1 to 6 queries of 30 / 6 heads,
// take 44 us, without it 115.
CachedPlan plan(const CachedAttnArgs& p, int cus) {
  CachedPlan pl;
  const int group = p.n_heads / p.n_kv_heads;
  // rows of the longest request, and of all in tiles of n rows
  int64_t most = 0;
  for (int r = 0; r < p.cq.n_req; ++r) most = std::max<int64_t>(most, (int64_t)(p.cq.cu[r + 1] - p.cq.cu[r]) * group);
  auto tiles = [&](int n) {
    int64_t k = 0;
    for (int r = 0; r < p.cq.n_req; ++r) k += ((int64_t)(p.cq.cu[r + 1] - p.cq.cu[r]) * group + n - 1) / n;
    return k;
  };
  pl.shape = p.dtype == DIT_F32 ? kF32 : most <= 32 ? kFew : kMany;
  pl.tile_rows = pl.shape == kF32 ? 16 : pl.shape == kFew ? 32 : 128;
  pl.unit_shift = pl.shape == kMany ? 6 : 7;
  pl.min_share = 256 >> pl.unit_shift;
  pl.extra = pl.shape == kMany ? 8 : 12;
  pl.shares = 0;
  const int64_t items = tiles(pl.tile_rows) * p.n_kv_heads;
  // workgroups that run at once, a multiple of the XCDs
  const int64_t cu = std::max(cus / kXcds * kXcds, kXcds), slots = (pl.shape == kMany ? 2 : 1) * cu;
  const int64_t n = ((int64_t)p.max_len + (1 << pl.unit_shift) - 1) >> pl.unit_shift;
  if (items > 0 && items < 8 * slots) {   // (of more, the last round is little)
    const int64_t units = items * (n + pl.extra);
    const int64_t shares = std::min(slots, ((units + pl.min_share - 1) / pl.min_share + kXcds - 1) / kXcds * kXcds);
    // us: of a workgroup beside its units; of a unit, with one workgroup per compute unit and with all; of joining
    const bool many = pl.shape == kMany;
    const double fixed = 9, alone = many ? 1.05 : pl.shape == kFew ? 0.5 : 1, full = many ? 1.75 : 1;
    const double joining = many ? 6 + 14.0 * shares / slots : 5;
    const int64_t rest = items % slots;
    const double whole = (items / slots) * (fixed + n * full) + (rest > 0 ? fixed + n * (rest > cu ? full : alone) : 0);
    const double share = std::max((double)units / shares, (double)pl.min_share);
    const double even = fixed + share * (shares > cu ? full : alone) + joining;
    if (even < whole) pl.shares = (int)shares;
  }
  // joining: up to 8 parts a row by one thread group, more by 2, 4 or 8 of the
  // workgroup's (1024 / head_dim) groups
  pl.merge_rows = 16;
  for (int g = 2; 4 * g * items <= pl.shares && pl.merge_rows > 1; g *= 2) pl.merge_rows = 1024 / p.head_dim / g;
  return pl;
}

}  // namespace

size_t cached_attention_ws(const CachedAttnArgs& p) {
  const CachedPlan pl = plan(p, cu_count());
  return (size_t)2 * pl.shares * pl.tile_rows * (p.head_dim + 2) * sizeof(float);
}

hipError_t launch_cached_attention(const CachedAttnArgs& p, void* ws, hipStream_t s) {
  if (p.q_gain && (p.head_dim != 128 || p.dtype != DIT_BF16)) return hipErrorInvalidValue;
  const CachedPlan pl = plan(p, cu_count());
  CachedWork w{};
  w.shares = pl.shares; w.unit_shift = pl.unit_shift; w.min_share = pl.min_share; w.extra = pl.extra;
  w.tile_rows = pl.tile_rows; w.merge_rows = pl.merge_rows;
  w.n_pages = p.n_pages; w.page_shift = p.page_shift; w.max_pages = p.max_pages; w.max_len = p.max_len;
  w.n_heads = p.n_heads; w.n_kv_heads = p.n_kv_heads; w.group = p.n_heads / p.n_kv_heads;
  w.q_stride = p.q_stride; w.o_stride = p.o_stride;
  w.k_pages = p.k_pages; w.v_pages = p.v_pages; w.k_scale = p.k_scale; w.v_scale = p.v_scale;
  w.table = p.table; w.lens = p.lens;
  w.q_gain = (const bf16*)p.q_gain; w.q_eps = p.q_eps;
  w.scale_log2 = p.scale * 1.4426950408889634f;
  w.part = (float*)ws;
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
    items += (int64_t)w.tiles[n] * p.n_kv_heads;
    if (items > kMaxItems) return hipErrorInvalidValue;
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
  const int grid = w.shares > 0 ? w.shares : per_xcd * kXcds;
  auto run = [&](auto hd, auto shares) {
    constexpr int HD = decltype(hd)::value;
    constexpr bool SHARES = decltype(shares)::value;
    const bf16* q = (const bf16*)p.q;
    bf16* o = (bf16*)p.o;
    if (pl.shape == kF32) cached_attn_f32<HD, SHARES><<<grid, 64 * kKeyWaves, 0, s>>>((const float*)p.q, (float*)p.o, w);
    else if (p.q_gain) {   // (the block's bf16 heads have 128 channels)
      if (pl.shape == kFew) cached_attn_few<128, true, SHARES><<<grid, 64 * kKeyWaves, 0, s>>>(q, o, w);
      else cached_attn_many<128, true, SHARES><<<grid, 256, 0, s>>>(q, o, w);
    } else if (pl.shape == kFew) cached_attn_few<HD, false, SHARES><<<grid, 64 * kKeyWaves, 0, s>>>(q, o, w);
    else cached_attn_many<HD, false, SHARES><<<grid, 256, 0, s>>>(q, o, w);
    if constexpr (SHARES) {
      const unsigned blocks = (unsigned)items * (pl.tile_rows / pl.merge_rows);
      if (pl.shape == kF32) cached_attn_merge<HD, float><<<blocks, 256, 0, s>>>((float*)p.o, w);
      else cached_attn_merge<HD, bf16><<<blocks, 256, 0, s>>>(o, w);
    }
  };
  auto run_hd = [&](auto hd) {
    if (w.shares > 0) run(hd, std::true_type{});
    else run(hd, std::false_type{});
  };
  if (p.head_dim == 64) run_hd(std::integral_constant<int, 64>{});
  else run_hd(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace dit
