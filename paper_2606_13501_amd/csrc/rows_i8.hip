// Rows in 8 bits, the operand of the Linears on 8-bit integers: a row y is
// written as int8 codes c and one fp32 scale s,
//   m = max(max|y|, 127 x 2^-100),  s = m / 127,  c = 127 y / m to nearest, ties to even,
// so that |c| <= 127 and y = c s within s / 2.  The row y is an activation or a
// weight as it is, the modulated LayerNorm of one, or the root-mean-square norm
// of a sum.  It is formed and kept in fp32: rounded to bf16 first, a value next
// to the largest would be off by 2^-9 of it before the codes round it by 2^-8.
// A row with a value that is not finite gets the scale NaN and codes of 0: what
// is computed from it is NaN.
//
// The kernels are bound by memory: a wave holds a row in registers from its one
// read to its one write (as the norms of 16-bit rows do).  In bf16, bytes in and
// out: modulated 75,600 x 5,120 206 us (5.6 TB/s) and 15,209 x 5,120 of four
// requests 52 us (4.5); sums and their RMS norm 32,760 x 5,120 184 us (6.4); rows
// of 13,824, 32,760 of them, 220 us (6.2).  These with other work between the
// calls; the comparisons below are of calls in a row, whose times differ from them
// by -3% to 15%.
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dit {

namespace {

constexpr float kLeastTop = 127.0f * 0x1p-100f;   // 127 / it = 2^100
constexpr int64_t kMaxGroups = 1 << 22;   // workgroups of a launch: 2^30 work-items; more rows take turns

// The wave's index, in a scalar register: so are its row's addresses then.
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// The largest magnitude so far, NaN once one has been seen (half an instruction a value).
__device__ __forceinline__ float top_of(float top, float v) { return __builtin_elementwise_maximum(top, fabsf(v)); }

// That of a wave: the bits of infinity and of every NaN are above the finite numbers'.
__device__ __forceinline__ uint32_t wave_top(float top) {
  uint32_t v = __float_as_uint(top) & 0x7FFFFFFFu;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, kWave));
  return v;
}

// How a row is scaled, from the bits of the largest magnitude of the numbers u
// that its codes are made from; the row itself is y = u f, 1 <= f < 2.
struct RowScale {
  float s;        // what is written
  float hi, lo;   // 127 / m in two parts, m the largest u
  bool fine;      // all values are finite
  __device__ explicit RowScale(uint32_t top, float f = 1.0f) {
    const float m = __uint_as_float(top), y = m * f;
    fine = y <= 0x1.fffffep127f;   // not of a NaN
    s = fine ? fmaxf(y, kLeastTop) / 127.0f : __uint_as_float(0x7FC00000u);
    const bool least = y < kLeastTop;
    hi = least ? f * 0x1p100f : 127.0f / m;
    lo = least ? 0.0f : fmaf(-hi, m, 127.0f) * hi * (1.0f / 127.0f);
  }
};

// VN codes as bytes: z + 1.5 x 2^23 leaves z, rounded to nearest even, in the
// low bits of the sum, two's complement.  The codes of rows as they are and of
// the RMS norm (TIES) take z = fl(y hi + y lo), which is 127 y / m rounded once to
// fp32 but for a part in 2^22 of the step between fp32 numbers: bf16 rows are often
// exactly in the middle between two codes (127 y / m = k + 1/2 for two numbers of 8
// bits, or of 16), and with 1 / s rounded such values went to either side (1 in
// 10,000 codes was off by one).  The modulated LayerNorm subtracts a mean, which
// leaves no such numbers but by chance: z = y hi inside the sum.
template <int VN> struct CodeVec;
template <> struct CodeVec<8> { typedef u32x2 type; };
template <> struct CodeVec<4> { typedef uint32_t type; };

template <bool TIES>
__device__ __forceinline__ uint32_t codes4(const float* y, const RowScale& q) {
  uint32_t u[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    u[e] = __float_as_uint(TIES ? fmaf(y[e], q.hi, y[e] * q.lo) + 12582912.0f : fmaf(y[e], q.hi, 12582912.0f));
  const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0C0C0400u);   // bytes: u0, u1, 0, 0
  const uint32_t hi = __builtin_amdgcn_perm(u[3], u[2], 0x04000C0Cu);   // 0, 0, u2, u3
  return q.fine ? lo | hi : 0u;
}

// Past the caches (32,760 rows of 13,824 215 us, 244 without) but for the RMS
// norm's, which leave with its sums (32,760 x 5,120 183 us, 192 past them).
template <int VN, bool TIES, bool CACHED = false>
__device__ __forceinline__ void store_codes(int8_t* at, const float (&y)[VN], const RowScale& q) {
  typename CodeVec<VN>::type o;
  if constexpr (VN == 8) {
    o[0] = codes4<TIES>(y, q);
    o[1] = codes4<TIES>(y + 4, q);
  } else {
    o = codes4<TIES>(y, q);
  }
  if (CACHED) *reinterpret_cast<typename CodeVec<VN>::type*>(at) = o;
  else __builtin_nontemporal_store(o, reinterpret_cast<typename CodeVec<VN>::type*>(at));
}

// The largest magnitude of a row held by WPR waves (their workgroup): each has
// `top` of its part.
template <int WPR>
__device__ __forceinline__ uint32_t row_top(float row) {
  uint32_t top = wave_top(row);
  if constexpr (WPR > 1) {
    __shared__ uint32_t tops[WPR];
    __syncthreads();   // the last row's are read
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WPR; ++w) top = max(top, tops[w]);
  }
  return top;
}

// y = x.  WPR waves per row (1: four rows per workgroup; 4: one).
template <typename T, int NVL, int WPR>
__global__ __launch_bounds__(256) void rows_i8_kernel(const T* __restrict__ x, int64_t x_stride, int8_t* __restrict__ codes,
                                                      int64_t codes_stride, float* __restrict__ scales, int64_t n_rows,
                                                      int width) {
  typedef typename Vec16<T>::type V;
  constexpr int VN = Vec16<T>::n, RPW = 4 / WPR;
  const int t = threadIdx.x & (64 * WPR - 1);   // thread of the row
  const int nv = width / VN;
  for (int64_t row = (int64_t)blockIdx.x * RPW + wave_id() / WPR; row < n_rows; row += (int64_t)gridDim.x * RPW) {
    const T* xr = x + row * x_stride;
    V v[NVL];
#pragma unroll
    for (int i = 0; i < NVL; ++i) {
      const int c = t + 64 * WPR * i;
      v[i] = c < nv ? __builtin_nontemporal_load(reinterpret_cast<const V*>(xr + c * VN)) : V{};
    }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < NVL; ++i)
#pragma unroll
      for (int e = 0; e < VN; ++e) top = top_of(top, to_f<T>(v[i][e]));
    const RowScale q(row_top<WPR>(top));
    if (t == 0) scales[row] = q.s;
    int8_t* cr = codes + row * codes_stride;
#pragma unroll
    for (int i = 0; i < NVL; ++i) {
      const int c = t + 64 * WPR * i;
      if (c < nv) {
        float y[VN];
#pragma unroll
        for (int e = 0; e < VN; ++e) y[e] = to_f<T>(v[i][e]);
        store_codes<VN, true>(cr + c * VN, y, q);
      }
    }
  }
}

// y = x for rows that registers do not hold: read twice, the second time from the caches.
template <typename T>
__global__ __launch_bounds__(256) void rows_i8_wide_kernel(const T* __restrict__ x, int64_t x_stride,
                                                           int8_t* __restrict__ codes, int64_t codes_stride,
                                                           float* __restrict__ scales, int64_t n_rows, int width) {
  typedef typename Vec16<T>::type V;
  constexpr int VN = Vec16<T>::n, U = 4;
  const int nv = width / VN;
  for (int64_t row = blockIdx.x; row < n_rows; row += gridDim.x) {
    const T* xr = x + row * x_stride;
    float top = 0.f;
    for (int c0 = threadIdx.x; c0 < nv; c0 += 256 * U) {
      V v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + 256 * u;
        v[u] = c < nv ? *reinterpret_cast<const V*>(xr + (int64_t)c * VN) : V{};
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < VN; ++e) top = top_of(top, to_f<T>(v[u][e]));
    }
    const RowScale q(row_top<4>(top));
    if (threadIdx.x == 0) scales[row] = q.s;
    int8_t* cr = codes + row * codes_stride;
    for (int c = threadIdx.x; c < nv; c += 256) {
      const V v = *reinterpret_cast<const V*>(xr + (int64_t)c * VN);
      float y[VN];
#pragma unroll
      for (int e = 0; e < VN; ++e) y[e] = to_f<T>(v[e]);
      store_codes<VN, true>(cr + (int64_t)c * VN, y, q);
    }
  }
}

// A wave's row y [NVL][VN] (zeros behind the row) times f as codes and scale.
template <int NVL, int VN, bool TIES, bool CACHED>
__device__ __forceinline__ void emit_codes(const float (&y)[NVL][VN], float f, int lane, int nv, int8_t* cr, float* scale) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < NVL; ++i)
#pragma unroll
    for (int e = 0; e < VN; ++e) top = top_of(top, y[i][e]);
  const RowScale q(wave_top(top), f);
  if (lane == 0) *scale = q.s;
#pragma unroll
  for (int i = 0; i < NVL; ++i)
    if (lane + 64 * i < nv) store_codes<VN, TIES, CACHED>(cr + (lane + 64 * i) * VN, y[i], q);
}

// y = LN(x) (1 + scale) + shift, a row per wave, four rows per workgroup and
// turn.  The statistics are those of the kernel that writes y in the rows' own
// type, in the same order, and so is y.  The workgroups stay resident and keep
// the vectors of a request in LDS from turn to turn (1 + scale and shift, 8 bytes
// a column): staged for every four rows, their reads from the L2 were four times
// the rows' bytes.  A turn over several requests' rows takes one after the other.
//
// Workgroups per compute unit (waves per SIMD), by the registers of a row in both
// forms and what goes with it, so that no instance spills (75,600 x 5,120 in bf16
// with 2, 3 and 4: 250, 235 and 493 us, 15,209 rows of it 58, 54 and 105).  Rows in
// fp32 lose by the largest number that fits (40,000 x 3,584 with 2 and 3: 121 and
// 125 us).  LDS holds as many.
template <typename T, int NVL>
constexpr int modulate_resident() {
  constexpr int registers = NVL * (4 + Vec16<T>::n) + 35;
  return registers <= 100 ? 4 : registers <= (sizeof(T) == 2 ? 155 : 140) ? 3 : 2;
}

template <typename T, int NVL>
__global__ __launch_bounds__(256, (modulate_resident<T, NVL>())) void modulate_i8_kernel(
    const T* __restrict__ x, int8_t* __restrict__ codes, float* __restrict__ scales, int64_t n_rows, int hidden, float eps,
    const float* __restrict__ shift, const float* __restrict__ scale, int64_t mod_stride, ReqTable req) {
  typedef typename Vec16<T>::type V;
  constexpr int VN = Vec16<T>::n, G = VN / 4;
  extern __shared__ f32x4 smod[];   // hidden / 4 vectors of 1 + scale, then of shift: vector G c + g at g nv + c
  const int lane = threadIdx.x & 63;
  const int nv = hidden / VN, h4 = hidden / 4;
  int kept = -1;                    // the request whose vectors are in LDS
  for (int64_t r0 = (int64_t)blockIdx.x * 4; r0 < n_rows; r0 += (int64_t)gridDim.x * 4) {
    const int64_t row = min(r0 + wave_id(), n_rows - 1);   // behind the last: the last once more
    V v[NVL];
#pragma unroll
    for (int i = 0; i < NVL; ++i) {
      const int c = lane + 64 * i;
      v[i] = c < nv ? __builtin_nontemporal_load(reinterpret_cast<const V*>(x + row * hidden + c * VN)) : V{};
    }
    const int mine = find_req(req.cu, req.n_req, (int)row);
    const int last = find_req(req.cu, req.n_req, (int)(min(r0 + 4, n_rows) - 1));
    for (int r = find_req(req.cu, req.n_req, (int)r0); r <= last; ++r) {   // nearly always one
      if (req.cu[r + 1] == req.cu[r]) continue;
      if (r != kept) {
        kept = r;
        __syncthreads();   // the former vectors are read
        const f32x4* sc = reinterpret_cast<const f32x4*>(scale + (int64_t)r * mod_stride);
        const f32x4* sh = reinterpret_cast<const f32x4*>(shift + (int64_t)r * mod_stride);
        for (int at = threadIdx.x; at < h4; at += 256) {
          const int i = G * (at % nv) + at / nv;
          f32x4 m = sc[i];
#pragma unroll
          for (int u = 0; u < 4; ++u) m[u] = 1.0f + m[u];
          smod[at] = m;
          smod[h4 + at] = sh[i];
        }
        __syncthreads();
      }
      if (mine != r) continue;
      // inside this loop, and hidden from the compiler, which would hold the
      // row in fp32 beside v and y from before it on
#pragma unroll
      for (int i = 0; i < NVL; ++i) asm volatile("" : "+v"(v[i]));
      float mean, rstd;
      row_stats<T, NVL>(v, lane, nv, hidden, eps, mean, rstd);
#pragma unroll
      for (int i = 0; i < NVL; ++i) asm volatile("" : "+v"(v[i]));
      float y[NVL][VN];
      // the lane hidden too: the places in LDS and memory that depend on it would be formed before the rows, all of them,
      // and spilled in wide rows (40,000 x 8,192 216 us, 173 so)
      int el = lane;
      asm volatile("" : "+v"(el));
      el &= 63;
#pragma unroll
      for (int i = 0; i < NVL; ++i) {
        const int c = el + 64 * i;
        const bool in = i < NVL - 2 || c < nv;   // (counts over 8 are rounded up to even ones)
        // behind the row, y is zero: with its mean, mean * rstd times the zeros there may be NaN though no value of the row is
        const float mu = in ? mean : 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          f32x4 m4{}, a4{};
          if (in) {
            m4 = smod[g * nv + c];
            a4 = smod[h4 + g * nv + c];
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) y[i][4 * g + u] = fmaf((to_f<T>(v[i][4 * g + u]) - mu) * rstd, m4[u], a4[u]);
        }
        // all of the request's vectors asked for at once do not fit the registers: these values before the next ones
        if (i % 2 == 1) {
#pragma unroll
          for (int e = 0; e < VN; ++e) asm volatile("" : "+v"(y[i - 1][e]), "+v"(y[i][e]) :: "memory");
        }
      }
      emit_codes<NVL, VN, false, false>(y, 1.0f, el, nv, codes + row * hidden, scales + row);
    }
  }
}

// sum = x + z rounded to T (z NULL: x itself), y = sum / sqrt(mean(sum^2) + eps)
// * gain, a row per wave.  The norm is that of the rounded sum, which is what
// the residual stream goes on with.  sum may be x or z, and out x or z: a row
// is read by the wave that writes it, before.
//
// 1 / rms is a factor of the whole row, so a code is that of sum * gain: a product
// of two bf16 numbers, which fp32 holds whole (above 2^-126).  Formed from y, whose
// two roundings move it, half of the values in the middle between two codes (14 in
// a million) got the odd one.
template <typename T, int NVL>
__global__ __launch_bounds__(256) void add_rms_kernel(const T* x, const T* z, const T* __restrict__ gain, T* sum, T* out,
                                                      int8_t* __restrict__ codes, float* __restrict__ scales, int64_t n_rows,
                                                      int hidden, float eps) {
  typedef typename Vec16<T>::type V;
  constexpr int VN = Vec16<T>::n;
  const int lane = threadIdx.x & 63;
  const int nv = hidden / VN;
  for (int64_t row = (int64_t)blockIdx.x * 4 + wave_id(); row < n_rows; row += (int64_t)gridDim.x * 4) {
    const int64_t at = row * hidden;
    V v[NVL];
#pragma unroll
    for (int i = 0; i < NVL; ++i) {
      const int c = lane + 64 * i;
      v[i] = c < nv ? __builtin_nontemporal_load(reinterpret_cast<const V*>(x + at + c * VN)) : V{};
    }
    if (z) {
      V w[NVL];
#pragma unroll
      for (int i = 0; i < NVL; ++i) {
        const int c = lane + 64 * i;
        w[i] = c < nv ? __builtin_nontemporal_load(reinterpret_cast<const V*>(z + at + c * VN)) : V{};
      }
#pragma unroll
      for (int i = 0; i < NVL; ++i) {
        const int c = lane + 64 * i;
#pragma unroll
        for (int e = 0; e < VN; ++e) v[i][e] = from_f<T>(to_f<T>(v[i][e]) + to_f<T>(w[i][e]));
        if (c < nv) __builtin_nontemporal_store(v[i], reinterpret_cast<V*>(sum + at + c * VN));
      }
    }
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < NVL; ++i)
#pragma unroll
      for (int e = 0; e < VN; ++e) {
        const float f = to_f<T>(v[i][e]);
        sq = fmaf(f, f, sq);
      }
    const float rs = rsqrtf(wave_sum(sq) / hidden + eps);
    if (out) {
#pragma unroll
      for (int i = 0; i < NVL; ++i) {
        const int c = lane + 64 * i;
        if (c < nv) {
          const V g = *reinterpret_cast<const V*>(gain + c * VN);
          V o;
#pragma unroll
          for (int e = 0; e < VN; ++e) o[e] = from_f<T>(to_f<T>(v[i][e]) * rs * to_f<T>(g[e]));
          __builtin_nontemporal_store(o, reinterpret_cast<V*>(out + at + c * VN));
        }
      }
    }
    if (codes) {
      // 1 / rms = p f, p a power of two: u = (sum p) gain is exact in bf16.  Behind the row it is zero (or NaN, where p is
      // not finite and the whole row is not).
      const float p = __uint_as_float(__float_as_uint(rs) & 0x7F800000u);
      const float f = __uint_as_float((__float_as_uint(rs) & 0x007FFFFFu) | 0x3F800000u);
      float u[NVL][VN];
#pragma unroll
      for (int i = 0; i < NVL; ++i) {
        const int c = lane + 64 * i;
        const V g = c < nv ? *reinterpret_cast<const V*>(gain + c * VN) : V{};
#pragma unroll
        for (int e = 0; e < VN; ++e) u[i][e] = to_f<T>(v[i][e]) * p * to_f<T>(g[e]);
      }
      emit_codes<NVL, VN, true, true>(u, f, lane, nv, codes + at, scales + row);
    }
  }
}

unsigned groups(int64_t n) { return (unsigned)(n < kMaxGroups ? n : kMaxGroups); }

template <typename T, int NVL>
hipError_t norm_nvl(const RowsI8Args& p, hipStream_t s) {
  const unsigned grid = groups((p.n_rows + 3) / 4);
  if (p.op == RowOp::kModulate)
    modulate_i8_kernel<T, NVL><<<std::min(grid, (unsigned)(modulate_resident<T, NVL>() * cu_count())), 256, (size_t)p.width * 8, s>>>((const T*)p.x, p.codes, p.scales, p.n_rows, p.width,
                                                                       p.eps, p.shift, p.scale, p.mod_stride, p.req);
  else if (p.op == RowOp::kRms)
    add_rms_kernel<T, NVL><<<grid, 256, 0, s>>>((const T*)p.x, (const T*)p.z, (const T*)p.gain, (T*)p.sum, (T*)p.out,
                                                p.codes, p.scales, p.n_rows, p.width, p.eps);
  else
    rows_i8_kernel<T, NVL, 1><<<grid, 256, 0, s>>>((const T*)p.x, p.x_stride, p.codes, p.codes_stride, p.scales, p.n_rows,
                                                   p.width);
  return hipGetLastError();
}

template <typename T, int NVL>
hipError_t rows_wg(const RowsI8Args& p, hipStream_t s) {
  rows_i8_kernel<T, NVL, 4><<<groups(p.n_rows), 256, 0, s>>>((const T*)p.x, p.x_stride, p.codes, p.codes_stride, p.scales,
                                                             p.n_rows, p.width);
  return hipGetLastError();
}

template <typename T>
hipError_t rows_typed(const RowsI8Args& p, hipStream_t s) {
  const int nv = p.width / Vec16<T>::n;
  switch ((nv + 63) / 64) {   // 16-byte vectors of a lane
    case 1: return norm_nvl<T, 1>(p, s);
    case 2: return norm_nvl<T, 2>(p, s);
    case 3: return norm_nvl<T, 3>(p, s);
    case 4: return norm_nvl<T, 4>(p, s);
    case 5: return norm_nvl<T, 5>(p, s);
    case 6: return norm_nvl<T, 6>(p, s);
    case 7: return norm_nvl<T, 7>(p, s);
    case 8: return norm_nvl<T, 8>(p, s);
    case 9: case 10: return norm_nvl<T, 10>(p, s);
    case 11: case 12: return norm_nvl<T, 12>(p, s);
    case 13: case 14: return norm_nvl<T, 14>(p, s);
    case 15: case 16: return norm_nvl<T, 16>(p, s);
    default: break;
  }
  if (p.op != RowOp::kRows) return hipErrorInvalidValue;
  switch ((nv + 255) / 256) {
    case 5: return rows_wg<T, 5>(p, s);
    case 6: return rows_wg<T, 6>(p, s);
    case 7: return rows_wg<T, 7>(p, s);
    case 8: return rows_wg<T, 8>(p, s);
    case 9: case 10: case 11: case 12: return rows_wg<T, 12>(p, s);
    case 13: case 14: case 15: case 16: return rows_wg<T, 16>(p, s);
    default: break;
  }
  rows_i8_wide_kernel<T><<<groups(p.n_rows), 256, 0, s>>>((const T*)p.x, p.x_stride, p.codes, p.codes_stride, p.scales,
                                                          p.n_rows, p.width);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rows_i8(const RowsI8Args& p, hipStream_t s) {
  if (p.n_rows == 0) return hipSuccess;
  return p.dtype == DIT_BF16 ? rows_typed<bf16>(p, s) : rows_typed<float>(p, s);
}

}  // namespace dit
