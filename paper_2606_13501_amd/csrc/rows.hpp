// What the kernels that hold a row in the registers of a wave share: its
// vectors and its LayerNorm statistics.
#pragma once

#include "common.hpp"

namespace dit {

namespace {

template <typename T> struct Vec16;
template <> struct Vec16<bf16> { typedef bf16x8 type; static constexpr int n = 8; };
template <> struct Vec16<float> { typedef f32x4 type; static constexpr int n = 4; };

// Mean and 1 / sqrt(var + eps) of the wave's row v (NVL vectors per lane).
// The squares are accumulated with explicit fused multiply-adds, so every
// kernel that calls this rounds the statistics the same way.
template <typename T, int NVL, typename V>
__device__ __forceinline__ void row_stats(const V (&v)[NVL], int lane, int nv, int hidden, float eps, float& mean,
                                          float& rstd) {
  constexpr int VN = Vec16<T>::n;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NVL; ++i)
#pragma unroll
    for (int e = 0; e < VN; ++e) sum += to_f<T>(v[i][e]);
  mean = wave_sum(sum) / hidden;
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < NVL; ++i) {
    if (lane + 64 * i < nv) {
#pragma unroll
      for (int e = 0; e < VN; ++e) {
        const float d = to_f<T>(v[i][e]) - mean;
        sq = fmaf(d, d, sq);
      }
    }
  }
  rstd = rsqrtf(wave_sum(sq) / hidden + eps);
}

}  // namespace

}  // namespace dit
