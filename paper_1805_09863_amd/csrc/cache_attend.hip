// Attention of one new token a row over its cached slots.
//
// One pass with the running maximum m and sum s of a softmax: a slot of score x
// takes (m, s, o) to (m', s e^(m - m') + e^(x - m'), o e^(m - m') + e^(x - m') v).
#include "cache_common.hpp"

namespace kb {

__device__ __forceinline__ float wave_sum(float x) {
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

template <class T>
__global__ __launch_bounds__(64) void cache_attend_rows(AttendArgs a) {
  constexpr int M = kCacheMaxDim / 64;
  const int r = blockIdx.x / a.q_heads, h = blockIdx.x % a.q_heads, lane = threadIdx.x;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const CacheView& c = a.c;
  const int D = c.dim, s = cache_seq(c, a.seq, r);
  const int len = s < 0 ? 0 : min(a.length[r], min(a.max_len, c.cap));
  const int kv = h / (a.q_heads / c.heads);
  const T* q = (const T*)a.q + r * a.q_stride + (int64_t)h * D;
  float x[M], o[M] = {}, m = -FLT_MAX, sum = 0.f;
  for (int i = 0; i < M; ++i) x[i] = lane + 64 * i < D ? (float)q[lane + 64 * i] : 0.f;
  for (int t = 0; t < len; ++t) {
    const int row = cache_row(c, c.table + (int64_t)s * c.max_pages, kv, t);
    if (row < 0) continue;
    const T *k = (const T*)c.k + (int64_t)row * D, *v = (const T*)c.v + (int64_t)row * D;
    float dot = 0.f;
    for (int i = 0; i < M; ++i)
      if (lane + 64 * i < D) dot += x[i] * (float)k[lane + 64 * i];
    const float score = wave_sum(dot) * a.scale, top = fmaxf(m, score);
    const float keep = expf(m - top), p = expf(score - top);
    m = top;
    sum = sum * keep + p;
    for (int i = 0; i < M; ++i)
      if (lane + 64 * i < D) o[i] = o[i] * keep + p * (float)v[lane + 64 * i];
  }
  const float norm = sum > 0.f ? 1.f / sum : 0.f;
  for (int i = 0; i < M; ++i)
    if (lane + 64 * i < D) ((T*)a.out)[((int64_t)r * a.q_heads + h) * D + lane + 64 * i] = (T)(o[i] * norm);
  if (lane == 0 && a.lse) a.lse[(int64_t)r * a.q_heads + h] = sum > 0.f ? m + logf(sum) : -INFINITY;
}

template <class T>
__global__ __launch_bounds__(256) void cache_attend_weights(AttendArgs a) {
  const CacheView& c = a.c;
  const int r = blockIdx.x / c.heads, kv = blockIdx.x % c.heads, lane = threadIdx.x & 63;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int D = c.dim, s = cache_seq(c, a.seq, r), group = a.q_heads / c.heads;
  const int len = s < 0 ? 0 : min(a.length[r], min(a.max_len, c.cap));
  for (int t = threadIdx.x >> 6; t < len; t += 4) {
    const int row = cache_row(c, c.table + (int64_t)s * c.max_pages, kv, t);
    if (row < 0) continue;
    const T* k = (const T*)c.k + (int64_t)row * D;
    float p = 0.f;
    for (int g = 0; g < group; ++g) {
      const int h = kv * group + g;
      const T* q = (const T*)a.q + r * a.q_stride + (int64_t)h * D;
      float dot = 0.f;
      for (int i = lane; i < D; i += 64) dot += (float)q[i] * (float)k[i];
      p += expf(wave_sum(dot) * a.scale - a.lse[(int64_t)r * a.q_heads + h]);
    }
    const int64_t at = ((int64_t)r * c.heads + kv) * c.cap + t;
    if (lane == 0) a.weight_out[at] = (a.weight_in ? a.weight_in[at] : 0.f) + p;
  }
}

template <class T>
static hipError_t launch(const AttendArgs& a, hipStream_t st) {
  cache_attend_rows<T><<<dim3(a.R * a.q_heads), dim3(64), 0, st>>>(a);
  if (a.weight_out) cache_attend_weights<T><<<dim3(a.R * a.c.heads), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_attend(int bf16, const AttendArgs& a, hipStream_t st) {
  return bf16 ? launch<__bf16>(a, st) : launch<float>(a, st);
}

}  // namespace kb
