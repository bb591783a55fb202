// The kernels after the attention's pass over the cache (cache_attend.hpp): the join of a row's
// splits, and the probabilities that eviction goes by.
#include "cache_common.hpp"

namespace kb {

// One (row, query head): with M = max m_p, sum_p e^(m_p - M) (s_p, o_p) over the splits that its
// length has.  Threads: 4 values of the head each, the splits shared out over what remains.
template <class T>
__global__ __launch_bounds__(256) void cache_attend_join(AttendArgs a) {
  __shared__ float4 part[256];
  __shared__ float red[4], red2[4];
  const CacheView& c = a.c;
  const int64_t rh = blockIdx.x;
  const int r = (int)(rh / a.q_heads), tid = threadIdx.x;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int s = cache_seq(c, a.seq, r);
  const int len = s < 0 || c.pages == 0 ? 0 : max(0, min(a.length[r], min(a.max_len, c.cap)));
  const int P = (len + a.chunk - 1) / a.chunk;
  const float2* stat = a.part_s + rh * a.splits;
  float top = -FLT_MAX, total = 0.f;
  for (int p = tid; p < P; p += 256) top = fmaxf(top, stat[p].x);
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if ((tid & 63) == 0) red[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  for (int p = tid; p < P; p += 256) total += exp2_fast(stat[p].x - top) * stat[p].y;
  for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
  if ((tid & 63) == 0) red2[tid >> 6] = total;

  const int width = c.dim / 4, shares = 256 / width, mine = tid / width, d = tid % width * 4;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (mine < shares)
    for (int p = mine; p < P; p += shares) {
      const float f = exp2_fast(stat[p].x - top);
      const float4 x = *(const float4*)(a.part_o + (rh * a.splits + p) * c.dim + d);
      o.x += f * x.x, o.y += f * x.y, o.z += f * x.z, o.w += f * x.w;
    }
  part[tid] = o;
  __syncthreads();
  if (tid >= width) return;
  total = (red2[0] + red2[1]) + (red2[2] + red2[3]);
  for (int i = 1; i < shares; ++i) {
    const float4 x = part[i * width + tid];
    o.x += x.x, o.y += x.y, o.z += x.z, o.w += x.w;
  }
  const float norm = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
  const T y[4] = {(T)(o.x * norm), (T)(o.y * norm), (T)(o.z * norm), (T)(o.w * norm)};
  __builtin_memcpy(__builtin_assume_aligned((T*)a.out + rh * c.dim + d, 4 * sizeof(T)), y, sizeof y);
  if (tid == 0 && a.lse) a.lse[rh] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * (1.f / kL2E);
}

// weight_out = weight_in + sum over the sharing heads of e^(x - lse), from the stored scores.
__global__ __launch_bounds__(256) void cache_attend_weights(AttendArgs a) {
  const CacheView& c = a.c;
  const int r = blockIdx.x / c.heads, kv = blockIdx.x % c.heads, group = a.q_heads / c.heads;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int len = c.pages == 0 ? 0 : max(0, min(a.length[r], min(a.max_len, c.cap)));
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

hipError_t launch_cache_attend_bf16(const AttendArgs& a, hipStream_t st);
hipError_t launch_cache_attend_f32(const AttendArgs& a, hipStream_t st);

hipError_t launch_cache_attend(int bf16, const AttendArgs& a, hipStream_t st) {
  hipError_t e = bf16 ? launch_cache_attend_bf16(a, st) : launch_cache_attend_f32(a, st);
  if (e != hipSuccess) return e;
  if (a.splits > 1) {
    if (bf16)
      cache_attend_join<__bf16><<<dim3(a.R * a.q_heads), dim3(256), 0, st>>>(a);
    else
      cache_attend_join<float><<<dim3(a.R * a.q_heads), dim3(256), 0, st>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.weight_out) {
    cache_attend_weights<<<dim3(a.R * a.c.heads, min(64, (min(a.max_len, a.c.cap) + 255) / 256)), dim3(256), 0, st>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace kb
