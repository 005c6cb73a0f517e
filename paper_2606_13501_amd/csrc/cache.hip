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
// the table entry of its page.  Latency-bound: a few KB in and out, 2.9 us for one
// request of 77 tokens, 3.3 us for 64 of 1,560.
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
// read and one written per value; 5 x 1,560 tokens x 40 heads of 128 in bf16
// take 55 us, 4.4 TB/s.
//
// Keys: a thread holds 16 channels of a token, one 16-byte piece of the page;
// a wave's stores are 8 tokens x 16 bytes at 8 channel chunks.  Values: a
// thread holds 8 channels of 4 tokens, one dword of 8 pieces; its wave puts the
// pieces together in LDS and stores them 16 bytes per lane, whole KiB at a time.
// (With 2 channels of 16 tokens per thread, 4-byte loads, the values took twice
// as long as the keys: 5 x 1,560 tokens x 40 heads of 128 81 us.)
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
    constexpr int LANES = HD / 2;                 // lanes of a unit, the pieces of 16 tokens (g, f): 4 x HD / 8
    constexpr int UNITS = PAGE / 16;
    constexpr int PER = THREADS / LANES;          // units of one pass
    constexpr int N = (UNITS + PER - 1) / PER;
    __shared__ __attribute__((aligned(16))) u32x4 s_piece[PER][HD];
    const int mine = tid / LANES, i = tid % LANES / (HD / 8), c = tid % (HD / 8);
    T x[N][4][8];
    uint32_t top = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int u = n * PER + mine;
      const int t0 = 32 * (u / 2) + 4 * (u % 2) + 8 * i;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[n][j][k] = (T)0.f;
        if (t0 + j >= offset && t0 + j < offset + count) {   // (u >= UNITS: the token is past the page)
          load_n(src + (int64_t)(t0 + j - offset) * stride + 8 * c, x[n][j]);
#pragma unroll
          for (int k = 0; k < 8; ++k) top = max(top, finite_bits(to_f<T>(x[n][j][k])));
        }
      }
    }
    choose(top);
    const float inv = pow2(254 - byte), mul = old_mul();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int u = n * PER + mine;
      const int t0 = 32 * (u / 2) + 4 * (u % 2);   // the unit's tokens: t0 + 8 i + j
      // dword i of channel d's piece; pieces of 8 channels are dealt over the banks
#pragma unroll
      for (int k = 0; k < 8; ++k)
        reinterpret_cast<uint32_t*>(&s_piece[mine][8 * c + (k ^ (c & 7))])[i] =
            pack4(scaled(to_f<T>(x[n][0][k]), inv), scaled(to_f<T>(x[n][1][k]), inv), scaled(to_f<T>(x[n][2][k]), inv),
                  scaled(to_f<T>(x[n][3][k]), inv));
      __builtin_amdgcn_wave_barrier();             // (a unit's lanes are one wave's)
      const bool touched = u < UNITS && t0 < offset + count && !(t0 + 27 < offset && byte == old);
      const bool whole = t0 >= offset && t0 + 27 < offset + count;
      u32x4* out = reinterpret_cast<u32x4*>(dst + (u / 2) * (32 * HD) + (u % 2) * (HD * 16));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int d = tid % LANES + h * LANES;
        u32x4 w = s_piece[mine][(d & ~7) + ((d & 7) ^ (d / 8 & 7))];
        if (touched && !whole) {
          const u32x4 was = out[d];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t held = byte > old ? rescale4(was[e], mul) : was[e];
            uint32_t v = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int t = t0 + 8 * e + j;
              v |= (t < offset ? held : t < offset + count ? w[e] : was[e]) & (0xFFu << (8 * j));
            }
            w[e] = v;
          }
        }
        if (touched) out[d] = w;
      }
      __builtin_amdgcn_wave_barrier();
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
  const int blocks = p.n_runs > 0 ? (p.n_runs - 1) / 256 + 1 : 1;   // (n_runs + 255 may pass 32 bits)
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
