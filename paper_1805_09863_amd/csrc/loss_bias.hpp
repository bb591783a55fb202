// The gradient of the bias from the row tiles' sums of the dlogits.
#pragma once

#include "loss_common.hpp"

namespace kb {

// Workgroup wg of 1,024 threads: 64 words; 16 groups of 64 threads add up every 16th row's sums, then the groups'.
// `sums`: 1,024 floats of LDS.
__device__ __forceinline__ void sum_bias(const LossBiasArgs& a, int wg, float* sums) {
  const int x = threadIdx.x & 63, grp = threadIdx.x >> 6, v = wg * 64 + x;
  const int n = loss_row_tiles(*a.count, a.BN) * a.wave_rows;
  float s = 0.f;
  if (v < a.V) {
#pragma unroll 4
    for (int i = grp; i < n; i += 16) s += a.dbp[(size_t)i * a.ld + v];
  }
  sums[grp * 64 + x] = s;
  __syncthreads();
  if (grp > 0 || v >= a.V) return;
#pragma unroll
  for (int g = 1; g < 16; ++g) s += sums[g * 64 + x];
  a.db[v] = s;
}

}  // namespace kb
