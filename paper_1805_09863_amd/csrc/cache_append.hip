// Rotary positions and the append of new tokens to the attention cache.
//
// A pair (x, y) of a head turned by the angle a = pos * freq: (x cos a - y sin a,
// x sin a + y cos a), times the amplitude.
#include "cache_common.hpp"

namespace kb {

// cos and sin of pos * freq times the amplitude.  The angle is reduced in 64
// bits: at position 10^6 a float32 product is off by up to 0.03 radians.
__device__ __forceinline__ float2 turn_of(int pos, double freq, float amplitude) {
  const double quarters = (double)pos * freq * 0.63661977236758134308;  // 2 / pi
  const double whole = rint(quarters);
  float s, c;
  sincospif(0.5f * (float)(quarters - whole), &s, &c);
  const int n = (int)((long long)whole & 3);
  const float cs = (n & 1) ? s : c, sn = (n & 1) ? c : s;
  return make_float2(((n + 1) & 2) ? -amplitude * cs : amplitude * cs, (n & 2) ? -amplitude * sn : amplitude * sn);
}

template <class T>
__global__ __launch_bounds__(256) void cache_append_rows(AppendArgs a) {
  __shared__ float2 turn[kCacheMaxDim / 2];
  const int r = blockIdx.x;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const CacheView& c = a.c;
  const int D = c.dim, half = a.rot / 2;
  const int s = cache_seq(c, a.seq, r);
  const int slot = s < 0 || a.length[r] > c.cap ? -1 : a.length[r] - 1;
  const int pos = a.pos ? a.pos[r] : slot;
  for (int i = threadIdx.x; i < half; i += 256) turn[i] = turn_of(pos, a.freq[i], a.amplitude);
  __syncthreads();

  auto head = [&](const T* x, T* y) {
    for (int i = threadIdx.x; i < half; i += 256) {
      const int lo = a.interleaved ? 2 * i : i, hi = a.interleaved ? 2 * i + 1 : i + half;
      const float u = (float)x[lo], w = (float)x[hi];
      const float2 cs = turn[i];
      y[lo] = (T)(u * cs.x - w * cs.y);
      y[hi] = (T)(u * cs.y + w * cs.x);
    }
    for (int i = a.rot + threadIdx.x; i < D; i += 256) y[i] = x[i];
  };
  for (int h = 0; h < a.q_heads; ++h)
    head((const T*)a.q + r * a.q_stride + (int64_t)h * D, (T*)a.q_out + ((int64_t)r * a.q_heads + h) * D);
  if (slot < 0) return;
  for (int h = 0; h < c.heads; ++h) {
    const int row = cache_row(c, c.table + (int64_t)s * c.max_pages, h, slot);
    if (row < 0) return;
    head((const T*)a.k_new + r * a.k_stride + (int64_t)h * D, (T*)c.k + (int64_t)row * D);
    for (int i = threadIdx.x; i < D; i += 256)
      ((T*)c.v)[(int64_t)row * D + i] = ((const T*)a.v_new)[r * a.v_stride + (int64_t)h * D + i];
    const int64_t at = ((int64_t)s * c.heads + h) * c.cap + slot;
    if (threadIdx.x == 0 && a.position) a.position[at] = pos;
    if (threadIdx.x == 0 && a.weight) a.weight[at] = 0.f;
  }
}

hipError_t launch_cache_append(int bf16, const AppendArgs& a, hipStream_t st) {
  if (bf16)
    cache_append_rows<__bf16><<<dim3(a.R), dim3(256), 0, st>>>(a);
  else
    cache_append_rows<float><<<dim3(a.R), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace kb
