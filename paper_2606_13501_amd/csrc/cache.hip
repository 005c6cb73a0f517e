// The paged 8-bit key/value cache: page tables and the slot map from the
// requests' lengths, and the writer of the pages.
//
// Values are float8 e4m3 codes times one power of two per page and head (its
// biased exponent is the scale byte).  e4m3 keeps 4 significant bits whatever
// the power of two, so such a scale rounds no worse than a general one, a page
// that grows is brought to a larger scale without a second rounding (except
// of values below 2^-6 of the new scale), and the matrix instructions and
// conversions of gfx950 take the byte as it is.
#include "common.hpp"
#include "kernels.hpp"

namespace dit {

namespace {

// One launch: every workgroup scans the (at most 64) requests with its first
// wave, one lane a request, then each thread fills one run of the slot map and
// the table entry of its page.  Latency-bound: a few KB in and out.
__global__ __launch_bounds__(256) void cache_tables_kernel(CacheTablesArgs p) {
  __shared__ int s_b[kWave], s_a[kWave], s_row0[kWave], s_have[kWave], s_base[kWave], s_runs_end[kWave];
  const int tid = threadIdx.x;
  const int P = 1 << p.page_shift;
  if (tid < kWave) {
    const bool on = tid < p.n_req;
    const int b = on && p.lens_before ? p.lens_before[tid] : 0;
    const int a = on ? p.added[tid] : 0;
    const int64_t cap = (int64_t)p.max_pages << p.page_shift;
    // inclusive sums over the requests; 64 bits, as the lengths are the caller's device memory
    auto scan = [&](int64_t v) {
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int64_t below = __shfl_up(v, o, kWave);
        if (tid >= o) v += below;
      }
      return v;
    };
    const int64_t rows = a > 0 ? a : 0;
    const int64_t row0 = p.rows_per_req > 0 ? (int64_t)tid * p.rows_per_req : scan(rows) - rows;
    bool ok = on && a >= 0 && b >= 0 && (int64_t)b + a <= cap;
    ok = ok && (p.rows_per_req > 0 ? a <= p.rows_per_req : row0 + a <= p.n_rows);
    const int have = ok ? (int)(((int64_t)b + P - 1) >> p.page_shift) : 0;
    const int end = ok ? (int)(((int64_t)b + a + P - 1) >> p.page_shift) : 0;
    const int want = end - have;
    const int64_t upto = scan(want);
    const bool taken = ok && (want == 0 || upto <= p.n_free);
    const int touched = taken && a > 0 ? end - (b >> p.page_shift) : 0;
    const int64_t runs_end = scan(touched);   // at most n_runs (checked on the host), so it fits an int
    s_b[tid] = b;
    s_a[tid] = a;
    s_row0[tid] = (int)row0;
    s_have[tid] = have;
    s_base[tid] = taken ? (int)(upto - want) : 0;
    s_runs_end[tid] = (int)runs_end;
    if (blockIdx.x == 0) {
      if (on) p.lens[tid] = taken ? b + a : (int)min(max((int64_t)b, (int64_t)0), cap);
      const int64_t pages = scan(taken ? want : 0), refused = scan(on && !taken), tokens = scan(taken ? a : 0);
      if (tid == kWave - 1) {
        p.counts[0] = (int)pages;
        p.counts[1] = (int)runs_end;
        p.counts[2] = (int)refused;
        p.counts[3] = (int)tokens;
      }
    }
  }
  __syncthreads();
  const int i = blockIdx.x * 256 + tid;
  if (i >= p.n_runs) return;
  int4 run = {0, 0, 0, 0};
  if (i < s_runs_end[kWave - 1]) {
    int lo = 0, hi = kWave - 1;   // the first request whose runs end after i
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_runs_end[mid] > i) hi = mid; else lo = mid + 1;
    }
    const int b = s_b[lo], have = s_have[lo];
    const int nth = i - (lo > 0 ? s_runs_end[lo - 1] : 0);
    const int page_i = (b >> p.page_shift) + nth;
    int32_t* entry = p.table + (int64_t)lo * p.max_pages + page_i;
    const int page = page_i >= have ? p.free_pages[s_base[lo] + page_i - have] : *entry;
    if (page_i >= have) *entry = page;
    const int64_t start = (int64_t)page_i << p.page_shift;
    const int first = max((int64_t)b, start), last = min((int64_t)b + s_a[lo], start + P);
    run = {page, s_row0[lo] + (first - b), (int)(first - start), last - first};
  }
  reinterpret_cast<int4*>(p.runs)[i] = run;
}

// fp32 bits of the largest finite magnitude -> the smallest scale byte s with
// magnitude <= 448 * 2^(s - 127); 448 = 1.75 * 2^8.  Not below kCacheScaleMin,
// where a code's value would leave the normal range of bf16.
__device__ __forceinline__ int scale_byte(uint32_t top) {
  return max((int)(top >> 23) - 8 + ((top & 0x7FFFFF) > 0x600000), kCacheScaleMin);
}
__device__ __forceinline__ float pow2(int biased) { return __uint_as_float((uint32_t)biased << 23); }

// magnitude bits for the maximum; infinities and NaN do not count
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}
// value in units of the scale; an infinity has no e4m3 code and becomes NaN
__device__ __forceinline__ float scaled(float x, float inv) {
  return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : x * inv;
}
// four e4m3 codes, rounded to nearest even
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ uint32_t rescale4(uint32_t codes, float mul) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
  const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  return pack4(lo[0] * mul, lo[1] * mul, hi[0] * mul, hi[1] * mul);
}

template <typename T, int N>
__device__ __forceinline__ void load_n(const T* src, T (&x)[N]) {
  constexpr int B = N * sizeof(T);
  if constexpr (B % 16 == 0) {
#pragma unroll
    for (int i = 0; i < B / 16; ++i) reinterpret_cast<u32x4*>(x)[i] = reinterpret_cast<const u32x4*>(src)[i];
  } else if constexpr (B == 8) {
    *reinterpret_cast<u32x2*>(x) = *reinterpret_cast<const u32x2*>(src);
  } else {
    static_assert(B == 4, "4, 8 or 16 n bytes");
    *reinterpret_cast<uint32_t*>(x) = *reinterpret_cast<const uint32_t*>(src);
  }
}

// One workgroup writes the keys or the values of one run (the tokens that one
// call adds to one page) and one head.  The input is read once, into
// registers: the largest magnitude over the workgroup gives the scale, then
// the same registers are converted and stored.  HBM-bound: sizeof(T) bytes
// read and one written per value.
//
// Keys: a thread holds 16 channels of a token, one 16-byte piece of the page;
// a wave's stores are 8 tokens x 16 bytes at 8 channel chunks.  Values: a
// thread holds 2 channels of the 16 tokens of one piece, so the transpose
// happens in its registers; its two pieces lie side by side.
//
// A run that starts inside a page continues it: the scale does not get
// smaller, and where it grows the page's earlier codes are rewritten in the
// new scale.  Bytes behind the run are left as they were.
template <typename T, int HD, int PAGE>
__global__ __launch_bounds__(PAGE == 32 ? 128 : 256) void cache_store_kernel(CacheStoreArgs p) {
  constexpr int THREADS = PAGE == 32 ? 128 : 256;
  constexpr int WAVES = THREADS / kWave;
  const uint32_t item = blockIdx.y * gridDim.x + blockIdx.x;
  if (item >= p.n_items) return;
  const int head = item % p.n_kv_heads;
  const int rest = item / p.n_kv_heads;
  const bool is_v = rest & 1;
  const int4 run = reinterpret_cast<const int4*>(p.runs)[rest >> 1];
  const int page = run.x, row = run.y, offset = run.z, count = run.w;
  // the slot map is device memory: an entry outside the pool, the page or the rows is not written
  if (count <= 0 || offset < 0 || (int64_t)offset + count > PAGE || page < 0 || page >= p.n_pages || row < 0 ||
      (int64_t)row + count > p.n_rows)
    return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t slot = (int64_t)page * p.n_kv_heads + head;
  char* dst = (char*)(is_v ? p.v_pages : p.k_pages) + slot * (PAGE * HD);
  uint8_t* scale = (is_v ? p.v_scale : p.k_scale) + slot;
  const int64_t stride = is_v ? p.v_stride : p.k_stride;
  const T* src = (const T*)(is_v ? p.v : p.k) + (int64_t)row * stride + (int64_t)head * HD;

  __shared__ uint32_t s_top[WAVES];
  int byte, old = kCacheScaleMin;
  auto choose = [&](uint32_t top) __attribute__((always_inline)) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, kWave));
    if (lane == 0) s_top[wave] = top;
    if (offset > 0) old = min(max((int)*scale, kCacheScaleMin), kCacheScaleMax);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = max(top, s_top[w]);
    byte = max(scale_byte(top), old);
    if (tid == 0) *scale = (uint8_t)byte;
  };
  // multiplier of the page's earlier codes: 2^(old - byte), 0 where nothing of them is left (448 * 2^-31)
  auto old_mul = [&]() { return byte - old > 30 ? 0.f : pow2(127 + old - byte); };

  if (!is_v) {
    constexpr int N = PAGE * (HD / 16) / THREADS > 0 ? PAGE * (HD / 16) / THREADS : 1;
    static_assert(N * THREADS == PAGE * (HD / 16), "whole passes");
    T x[N][16];
    uint32_t top = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int e = n * THREADS + tid, t = e / (HD / 16), c = e % (HD / 16);
#pragma unroll
      for (int k = 0; k < 16; ++k) x[n][k] = (T)0.f;
      if (t >= offset && t < offset + count) {
        load_n(src + (int64_t)(t - offset) * stride + 16 * c, x[n]);
#pragma unroll
        for (int k = 0; k < 16; ++k) top = max(top, finite_bits(to_f<T>(x[n][k])));
      }
    }
    choose(top);
    const float inv = pow2(254 - byte), mul = old_mul();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int e = n * THREADS + tid, t = e / (HD / 16), c = e % (HD / 16);
      u32x4* out = reinterpret_cast<u32x4*>(dst + (t / 32) * (32 * HD) + c * 512 + (t % 32) * 16);
      u32x4 w;
      if (t >= offset && t < offset + count) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          w[k] = pack4(scaled(to_f<T>(x[n][4 * k]), inv), scaled(to_f<T>(x[n][4 * k + 1]), inv),
                       scaled(to_f<T>(x[n][4 * k + 2]), inv), scaled(to_f<T>(x[n][4 * k + 3]), inv));
        *out = w;
      } else if (t < offset && byte > old) {
        w = *out;
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = rescale4(w[k], mul);
        *out = w;
      }
    }
  } else {
    constexpr int PAIRS = HD / 2;                 // lanes of one piece row
    constexpr int UNITS = PAGE / 16;              // (group, f) pieces rows of the page
    constexpr int PER = THREADS / PAIRS;          // units of one pass
    constexpr int N = (UNITS + PER - 1) / PER;
    T x[N][16][2];
    uint32_t top = 0;
    const int d = 2 * (tid % PAIRS);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int u = n * PER + tid / PAIRS;
      // slot 4 i + j of unit (g, f) is token 32 g + 8 i + 4 f + j
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const int t = 32 * (u / 2) + 8 * (k / 4) + 4 * (u % 2) + k % 4;
        x[n][k][0] = x[n][k][1] = (T)0.f;
        if (t >= offset && t < offset + count) {   // (u >= UNITS: t is past the page)
          load_n(src + (int64_t)(t - offset) * stride + d, x[n][k]);
          top = max(top, max(finite_bits(to_f<T>(x[n][k][0])), finite_bits(to_f<T>(x[n][k][1]))));
        }
      }
    }
    choose(top);
    const float inv = pow2(254 - byte), mul = old_mul();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int u = n * PER + tid / PAIRS;
      if (u >= UNITS) continue;
      const int t0 = 32 * (u / 2) + 4 * (u % 2);   // tokens t0 .. t0 + 27 in steps of 8
      if (t0 >= offset + count || (t0 + 27 < offset && byte == old)) continue;
      u32x4* out = reinterpret_cast<u32x4*>(dst + (u / 2) * (32 * HD) + (u % 2) * (HD * 16) + d * 16);
      const bool whole = t0 >= offset && t0 + 27 < offset + count;
      u32x4 w[2];
      if (!whole) {
        w[0] = out[0];
        w[1] = out[1];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) f[j] = scaled(to_f<T>(x[n][4 * i + j][h]), inv);
          const uint32_t fresh = pack4(f[0], f[1], f[2], f[3]);
          if (whole) {
            w[h][i] = fresh;
          } else {
            const uint32_t held = byte > old ? rescale4(w[h][i], mul) : w[h][i];
            uint32_t v = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int t = t0 + 8 * i + j;
              const uint32_t from = t < offset ? held : t < offset + count ? fresh : w[h][i];
              v |= from & (0xFFu << (8 * j));
            }
            w[h][i] = v;
          }
        }
      }
      out[0] = w[0];
      out[1] = w[1];
    }
  }
}

template <typename T, int HD>
hipError_t store_page(const CacheStoreArgs& p, dim3 grid, hipStream_t s) {
  switch (p.page_tokens) {
    case 32: cache_store_kernel<T, HD, 32><<<grid, 128, 0, s>>>(p); break;
    case 64: cache_store_kernel<T, HD, 64><<<grid, 256, 0, s>>>(p); break;
    case 128: cache_store_kernel<T, HD, 128><<<grid, 256, 0, s>>>(p); break;
    case 256: cache_store_kernel<T, HD, 256><<<grid, 256, 0, s>>>(p); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_tables(const CacheTablesArgs& p, hipStream_t s) {
  const int blocks = p.n_runs > 0 ? (p.n_runs + 255) / 256 : 1;
  cache_tables_kernel<<<blocks, 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_cache_store(CacheStoreArgs p, int n_runs, hipStream_t s) {
  const int64_t items = (int64_t)n_runs * 2 * p.n_kv_heads;
  if (items == 0) return hipSuccess;
  if (items > 0x7FFFFFFF) return hipErrorInvalidValue;
  p.n_items = (uint32_t)items;
  // fewer than 2^32 work-items per grid dimension
  const unsigned nx = (unsigned)(items < (1 << 22) ? items : 1 << 22);
  const dim3 grid(nx, (unsigned)((items + nx - 1) / nx));
  if (p.dtype == DIT_BF16) return p.head_dim == 64 ? store_page<bf16, 64>(p, grid, s) : store_page<bf16, 128>(p, grid, s);
  return p.head_dim == 64 ? store_page<float, 64>(p, grid, s) : store_page<float, 128>(p, grid, s);
}

}  // namespace dit
