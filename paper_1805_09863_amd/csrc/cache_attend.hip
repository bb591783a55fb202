// The kernels after the attention's pass over the cache (cache_attend.hpp): the join of a row's
// splits, and the probabilities that eviction goes by.
#include "cache_common.hpp"

namespace kb {

// A (row, query head)'s partials: P of them, the i-th at at(i).
struct Splits {
  int64_t first;
  int P;
  __device__ __forceinline__ Splits(const AttendArgs& a, int64_t rh, int r) {
    const int s = cache_seq(a.c, a.seq, r), len = s < 0 ? 0 : max(0, min(a.length[r], a.max_len));
    first = rh * a.splits;
    P = (len + a.chunk - 1) / a.chunk;
  }
  __device__ __forceinline__ bool finished() const { return false; }
  __device__ __forceinline__ int64_t at(int i) const { return first + i; }
};

struct Shares {
  int64_t head;
  int b0, first, P;
  bool whole;
  __device__ __forceinline__ Shares(const AttendArgs& a, int64_t rh, int r) {
    const int group = a.q_heads / a.c.heads, h = (int)(rh - (int64_t)r * a.q_heads), in = h % group;
    const int hp = h / group * a.head_tiles + in / 16, rows = rows_of(a.R, a.n_dev);
    const int before = a.row_before[r], cost = a.row_before[r + 1] - before, all = a.row_before[rows];
    const AttendShares shares(all, a.c.heads * a.head_tiles, a.shares);
    const long long x = (long long)hp * all + before;
    b0 = shares.of(x);
    const int b1 = shares.of(x + cost - 1);
    whole = b0 == b1;
    head = in % 16;
    // the row's first share may end within the start, and its slots begin in the second or third; shares
    // of a row without slots hold none of it
    first = b0;
    while (first <= b1 && min(shares.begin(first + 1) - x, (long long)cost) <= AttendShares::kStart) ++first;
    P = b1 - first + 1;
  }
  __device__ __forceinline__ bool finished() const { return whole; }
  __device__ __forceinline__ int64_t at(int i) const {
    return AttendShares::partial(first + i, first + i == b0 ? 0 : 1) * 16 + head;
  }
};

// One (row, query head): with M = max m_p, sum_p e^(m_p - M) (s_p, o_p) over its partials.  A thread
// takes 4 values of the head and every SHARES-th partial; with one share a workgroup takes as many
// (row, head)s as fit.
template <class T, class Parts, bool ONE>
__global__ __launch_bounds__(256) void cache_attend_join(AttendArgs a) {
  __shared__ float4 part[ONE ? 1 : 256];
  __shared__ float part_sum[ONE ? 1 : 256], part_top[ONE ? 1 : 4];
  const CacheView& c = a.c;
  const int width = c.dim / 4, fit = 256 / width, mine = threadIdx.x / width, d = threadIdx.x % width * 4;
  const int shares = ONE ? 1 : fit, share = ONE ? 0 : mine;
  const int64_t rh = ONE ? (int64_t)blockIdx.x * fit + mine : blockIdx.x;
  const int r = (int)(rh / a.q_heads);
  if (r >= rows_of(a.R, a.n_dev)) return;
  const Parts parts(a, rh, r);
  if (parts.finished()) return;
  if (ONE && mine >= fit) return;
  const int P = parts.P;
  float top = -FLT_MAX, total = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  if constexpr (ONE) {
#pragma unroll 8
    for (int p = 0; p < P; ++p) top = fmaxf(top, a.part_s[parts.at(p)].x);
  } else {
    for (int p = threadIdx.x; p < P; p += 256) top = fmaxf(top, a.part_s[parts.at(p)].x);
    for (int i = 32; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
    if (threadIdx.x % 64 == 0) part_top[threadIdx.x / 64] = top;
    __syncthreads();
    top = fmaxf(fmaxf(part_top[0], part_top[1]), fmaxf(part_top[2], part_top[3]));
  }
  if (mine < fit)
#pragma unroll 4
    for (int p = share; p < P; p += shares) {
      const float2 stat = a.part_s[parts.at(p)];
      const float4 y = *(const float4*)(a.part_o + parts.at(p) * c.dim + d);
      const float f = exp2_fast(stat.x - top);
      total += f * stat.y;
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
  const float norm = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
  const T y[4] = {(T)(o[0] * norm), (T)(o[1] * norm), (T)(o[2] * norm), (T)(o[3] * norm)};
  __builtin_memcpy(__builtin_assume_aligned((T*)a.out + rh * c.dim + d, 4 * sizeof(T)), y, sizeof y);
  if (d == 0 && a.lse) a.lse[rh] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * (1.f / kL2E);
}

// weight_out = weight_in + sum over the sharing heads of e^(x - lse), from the stored scores, 4 slots a
// thread.
__global__ __launch_bounds__(256) void cache_attend_weights(AttendArgs a) {
  const CacheView& c = a.c;
  const int r = blockIdx.x / c.heads, kv = blockIdx.x % c.heads, group = a.q_heads / c.heads;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int len = max(0, min(a.length[r], a.max_len));
  const int64_t rh = (int64_t)r * a.q_heads + kv * group, at = ((int64_t)r * c.heads + kv) * c.cap;
  for (int t = (blockIdx.y * 256 + threadIdx.x) * 4; t < len; t += gridDim.y * 1024) {
    float p[4] = {0.f, 0.f, 0.f, 0.f}, old[4] = {0.f, 0.f, 0.f, 0.f};
    bool there[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      there[i] = t + i < len;
      if (a.weight_in && there[i]) old[i] = a.weight_in[at + t + i];
    }
#pragma unroll 4
    for (int h = 0; h < group; ++h) {
      const float4 y = *(const float4*)(a.scores + (rh + h) * a.score_ld + t);  // rows end at whole tiles
      const float x[4] = {y.x, y.y, y.z, y.w}, lse = a.lse[rh + h] * kL2E;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        there[i] &= x[i] != -INFINITY;  // a hole
        p[i] += exp2_fast(x[i] - lse);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (there[i]) a.weight_out[at + t + i] = old[i] + p[i];
  }
}

// Few (row, head)s may have many partials each, which are shared out; of many one thread a value walks them.
template <class T, class Parts>
static hipError_t launch_join(const AttendArgs& a, hipStream_t st) {
  const int pairs = a.R * a.q_heads, fit = 256 / (a.c.dim / 4);
  if (pairs > 2048)
    cache_attend_join<T, Parts, true><<<dim3((pairs + fit - 1) / fit), dim3(256), 0, st>>>(a);
  else
    cache_attend_join<T, Parts, false><<<dim3(pairs), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

template <class T>
static hipError_t launch_joins(const AttendArgs& a, hipStream_t st) {
  return a.shares > 0 ? launch_join<T, Shares>(a, st) : a.splits > 1 ? launch_join<T, Splits>(a, st) : hipSuccess;
}

hipError_t launch_cache_attend_bf16(const AttendArgs& a, hipStream_t st);
hipError_t launch_cache_attend_f32(const AttendArgs& a, hipStream_t st);

hipError_t launch_cache_attend(int bf16, const AttendArgs& a, hipStream_t st) {
  hipError_t e = bf16 ? launch_cache_attend_bf16(a, st) : launch_cache_attend_f32(a, st);
  if (e != hipSuccess) return e;
  e = bf16 ? launch_joins<__bf16>(a, st) : launch_joins<float>(a, st);
  if (e != hipSuccess) return e;
  if (a.weight_out) {
    // no more workgroups than the card starts in a few microseconds
    const int pairs = a.R * a.c.heads, blocks = max(1, min((a.max_len + 1023) / 1024, 4096 / pairs));
    cache_attend_weights<<<dim3(pairs, blocks), dim3(256), 0, st>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace kb
