// The kernels after the attention's pass over the cache (cache_attend.hpp): the join of a row's
// splits, and the probabilities that eviction goes by.
#include "cache_common.hpp"

namespace kb {

constexpr int kJoinOne = 8;  // splits that one thread a value walks

// One (row, query head): with M = max m_p, sum_p e^(m_p - M) (s_p, o_p) over the splits that its
// length has.  A thread takes 4 values of the head and every SHARES-th split; with one share a
// workgroup takes as many (row, head)s as fit.
template <class T, bool ONE>
__global__ __launch_bounds__(256) void cache_attend_join(AttendArgs a) {
  __shared__ float4 part[ONE ? 1 : 256];
  __shared__ float part_sum[ONE ? 1 : 256], part_top[ONE ? 1 : 4];
  const CacheView& c = a.c;
  const int width = c.dim / 4, fit = 256 / width, mine = threadIdx.x / width, d = threadIdx.x % width * 4;
  const int shares = ONE ? 1 : fit, share = ONE ? 0 : mine;
  const int64_t rh = ONE ? (int64_t)blockIdx.x * fit + mine : blockIdx.x;
  const int r = (int)(rh / a.q_heads);
  const bool there = mine < fit && r < rows_of(a.R, a.n_dev);
  const int s = there ? cache_seq(c, a.seq, r) : -1;
  const int len = s < 0 ? 0 : max(0, min(a.length[r], a.max_len));
  const int P = (len + a.chunk - 1) / a.chunk;
  const float2* stat = a.part_s + rh * a.splits;
  const float* x = a.part_o + rh * a.splits * c.dim + d;
  float top = -FLT_MAX, total = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  if constexpr (ONE) {
#pragma unroll
    for (int p = 0; p < kJoinOne; ++p) top = p < P ? fmaxf(top, stat[p].x) : top;
  } else {
    for (int p = threadIdx.x; p < P; p += 256) top = fmaxf(top, stat[p].x);
    for (int i = 32; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
    if (threadIdx.x % 64 == 0) part_top[threadIdx.x / 64] = top;
    __syncthreads();
    top = fmaxf(fmaxf(part_top[0], part_top[1]), fmaxf(part_top[2], part_top[3]));
  }
#pragma unroll 4
  for (int p = share; p < P; p += shares) {
    const float f = exp2_fast(stat[p].x - top);
    const float4 y = *(const float4*)(x + (int64_t)p * c.dim);
    total += f * stat[p].y;
    o[0] += f * y.x, o[1] += f * y.y, o[2] += f * y.z, o[3] += f * y.w;
  }
  if constexpr (!ONE) {
    part[threadIdx.x] = make_float4(o[0], o[1], o[2], o[3]);
    part_sum[threadIdx.x] = total;
    __syncthreads();
    if (mine > 0) return;
    for (int i = 1; i < shares; ++i) {
      const float4 y = part[i * width + threadIdx.x];
      total += part_sum[i * width + threadIdx.x];
      o[0] += y.x, o[1] += y.y, o[2] += y.z, o[3] += y.w;
    }
  }
  if (!there) return;
  const float norm = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
  const T y[4] = {(T)(o[0] * norm), (T)(o[1] * norm), (T)(o[2] * norm), (T)(o[3] * norm)};
  __builtin_memcpy(__builtin_assume_aligned((T*)a.out + rh * c.dim + d, 4 * sizeof(T)), y, sizeof y);
  if (d == 0 && a.lse) a.lse[rh] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * (1.f / kL2E);
}

// weight_out = weight_in + sum over the sharing heads of e^(x - lse), from the stored scores.
__global__ __launch_bounds__(256) void cache_attend_weights(AttendArgs a) {
  const CacheView& c = a.c;
  const int r = blockIdx.x / c.heads, kv = blockIdx.x % c.heads, group = a.q_heads / c.heads;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int len = max(0, min(a.length[r], a.max_len));
  const int64_t rh = (int64_t)r * a.q_heads + kv * group, at = ((int64_t)r * c.heads + kv) * c.cap;
  for (int t = blockIdx.y * 256 + threadIdx.x; t < len; t += gridDim.y * 256) {
    float p = 0.f;
    bool there = true;
    for (int h = 0; h < group; ++h) {
      const float x = a.scores[(rh + h) * a.score_ld + t];
      there = there && x != -INFINITY;  // a hole
      p += exp2_fast(x - a.lse[rh + h] * kL2E);
    }
    if (there) a.weight_out[at + t] = (a.weight_in ? a.weight_in[at + t] : 0.f) + p;
  }
}

// Many splits of few (row, head)s are shared out; otherwise one thread a value walks them.
template <class T>
static hipError_t launch_join(const AttendArgs& a, hipStream_t st) {
  const int pairs = a.R * a.q_heads, fit = 256 / (a.c.dim / 4);
  if (a.splits <= kJoinOne)
    cache_attend_join<T, true><<<dim3((pairs + fit - 1) / fit), dim3(256), 0, st>>>(a);
  else
    cache_attend_join<T, false><<<dim3(pairs), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_attend_bf16(const AttendArgs& a, hipStream_t st);
hipError_t launch_cache_attend_f32(const AttendArgs& a, hipStream_t st);

hipError_t launch_cache_attend(int bf16, const AttendArgs& a, hipStream_t st) {
  hipError_t e = bf16 ? launch_cache_attend_bf16(a, st) : launch_cache_attend_f32(a, st);
  if (e != hipSuccess) return e;
  if (a.splits > 1) {
    e = bf16 ? launch_join<__bf16>(a, st) : launch_join<float>(a, st);
    if (e != hipSuccess) return e;
  }
  if (a.weight_out) {
    cache_attend_weights<<<dim3(a.R * a.c.heads, min(64, (a.max_len + 255) / 256)), dim3(256), 0, st>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace kb
