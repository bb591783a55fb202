// What follows the attention's pass over the cache (cache_attend.hpp), in one launch: the join of a
// row's partials, and the probabilities that eviction goes by.
#include "cache_common.hpp"

namespace kb {

// The partials of row r's ht-th 16 query heads of key-value head kv: P of them, the i-th of the tile's head
// n at at(i, n); or the pass has finished the row.
struct Whole {
  static constexpr int P = 0;
  __device__ __forceinline__ Whole(const AttendArgs&, int, int, int) {}
  __device__ __forceinline__ bool finished() const { return true; }
  __device__ __forceinline__ int64_t at(int, int) const { return 0; }
};

struct Splits {
  int64_t first;
  int splits, P;
  __device__ __forceinline__ Splits(const AttendArgs& a, int r, int kv, int ht) : splits(a.splits) {
    const int s = cache_seq(a.c, a.seq, r), len = s < 0 ? 0 : max(0, min(a.length[r], a.max_len));
    first = ((int64_t)r * a.q_heads + kv * (a.q_heads / a.c.heads) + ht * 16) * splits;
    P = (len + a.chunk - 1) / a.chunk;
  }
  __device__ __forceinline__ bool finished() const { return false; }
  __device__ __forceinline__ int64_t at(int i, int n) const { return first + (int64_t)n * splits + i; }
};

struct Shares {
  int b0, first, P;
  bool whole;
  __device__ __forceinline__ Shares(const AttendArgs& a, int r, int kv, int ht) {
    const int before = a.row_before[r], cost = a.row_before[r + 1] - before, all = a.row_before[rows_of(a.R, a.n_dev)];
    const AttendShares shares(all, a.c.heads * a.head_tiles);
    const long long x = (long long)(kv * a.head_tiles + ht) * all + before;
    b0 = shares.of(x);
    const int b1 = shares.of(x + cost - 1);
    whole = b0 == b1;
    // the row's first share may end within the start, and its slots begin in the second; shares of a row
    // without slots hold none of it
    first = b0;
    while (first <= b1 && min(shares.begin(first + 1) - x, (long long)cost) <= AttendShares::kStart) ++first;
    P = b1 - first + 1;
  }
  __device__ __forceinline__ bool finished() const { return whole; }
  __device__ __forceinline__ int64_t at(int i, int n) const {
    return AttendShares::partial(first + i, first + i == b0 ? 0 : 1) * 16 + n;
  }
};

// One (row, query head): with M = max m_p, sum_p e^(m_p - M) (s_p, o_p) over its partials.  A thread
// takes 4 values of the head and, of many partials of few (row, head)s, every so many-th; with ONE all of
// them, and a workgroup takes as many (row, head)s as fit.
template <class T, class Parts, bool ONE>
__device__ __forceinline__ void join(const AttendArgs& a, int block) {
  __shared__ float4 part[ONE ? 1 : 256];
  __shared__ float part_sum[ONE ? 1 : 256], part_top[ONE ? 1 : 4];
  const CacheView& c = a.c;
  const int width = c.dim / 4, fit = 256 / width, mine = threadIdx.x / width, d = threadIdx.x % width * 4;
  const int shares = ONE ? 1 : fit, share = ONE ? 0 : mine;
  const int64_t rh = ONE ? (int64_t)block * fit + mine : block;
  const int r = (int)(rh / a.q_heads), h = (int)(rh - (int64_t)r * a.q_heads);
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int group = a.q_heads / c.heads, kv = h / group, n = (h - kv * group) % 16;
  const Parts parts(a, r, kv, (h - kv * group) / 16);
  if (parts.finished()) return;
  if (ONE && mine >= fit) return;
  const int P = parts.P;
  float top = -FLT_MAX, total = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  if constexpr (ONE) {
#pragma unroll 8
    for (int p = 0; p < P; ++p) top = fmaxf(top, a.part_s[parts.at(p, n)].x);
  } else {
    for (int p = threadIdx.x; p < P; p += 256) top = fmaxf(top, a.part_s[parts.at(p, n)].x);
    for (int i = 32; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
    if (threadIdx.x % 64 == 0) part_top[threadIdx.x / 64] = top;
    __syncthreads();
    top = fmaxf(fmaxf(part_top[0], part_top[1]), fmaxf(part_top[2], part_top[3]));
  }
  if (mine < fit)
#pragma unroll 4
    for (int p = share; p < P; p += shares) {
      const float2 stat = a.part_s[parts.at(p, n)];
      const float4 y = *(const float4*)(a.part_o + parts.at(p, n) * c.dim + d);
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

// One (row, key-value head): weight_out = weight_in + sum over the sharing query heads of e^(x - m) / sum, from
// the stored scores, 4 slots a thread, 16 query heads at a time.  The maxima m and sums of those that the pass has
// not finished are worked out again from the partials, a wave a head: the join need not have run.  (x less the
// log-sum-exp would cost a rounding of that one's size in every weight.)
template <class Parts>
__device__ __forceinline__ void weights(const AttendArgs& a, int block) {
  __shared__ float2 stat[16];  // m, 1 / sum
  const CacheView& c = a.c;
  const int pairs = a.R * c.heads, y = block / pairs, pair = block - y * pairs;  // short rows have no later blocks
  const int r = pair / c.heads, kv = pair - r * c.heads, group = a.q_heads / c.heads, lane = threadIdx.x & 63;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int len = max(0, min(a.length[r], a.max_len));
  if (y * 1024 >= len) return;
  const int64_t at = ((int64_t)r * c.heads + kv) * c.cap;
  for (int ht = 0; ht < a.head_tiles; ++ht) {
    const int64_t rh = (int64_t)r * a.q_heads + kv * group + ht * 16;
    const int nh = min(16, group - ht * 16);
    const Parts parts(a, r, kv, ht);
    for (int n = threadIdx.x >> 6; n < nh; n += 4) {
      if (parts.finished()) {
        if (lane == 0) stat[n] = a.finished[rh + n];
        continue;
      }
      float top = -FLT_MAX, total = 0.f;
      for (int p = lane; p < parts.P; p += 64) top = fmaxf(top, a.part_s[parts.at(p, n)].x);
      for (int i = 32; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
      for (int p = lane; p < parts.P; p += 64) {
        const float2 s = a.part_s[parts.at(p, n)];
        total += exp2_fast(s.x - top) * s.y;
      }
      for (int i = 32; i > 0; i >>= 1) total += __shfl_xor(total, i);
      if (lane == 0) stat[n] = make_float2(top, 1.f / total);
    }
    __syncthreads();
    const float* in = ht == 0 ? a.weight_in : a.weight_out;  // later heads add to what this thread has written
    for (int t = (y * 256 + threadIdx.x) * 4; t < len; t += a.weight_blocks * 1024) {
      float p[4] = {0.f, 0.f, 0.f, 0.f}, old[4] = {0.f, 0.f, 0.f, 0.f};
      bool there[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        there[i] = t + i < len;
        if (in && there[i]) old[i] = in[at + t + i];
      }
#pragma unroll 4
      for (int n = 0; n < nh; ++n) {
        const float4 z = *(const float4*)(a.scores + (rh + n) * a.score_ld + t);  // rows end at whole tiles
        const float2 s = stat[n];
        const float x[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          there[i] &= x[i] != -INFINITY;  // a hole
          p[i] += exp2_fast(x[i] - s.x) * s.y;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (there[i]) a.weight_out[at + t + i] = old[i] + p[i];
    }
    __syncthreads();
  }
}

template <class T, class Parts, bool ONE>
__global__ __launch_bounds__(256) void cache_attend_finish(AttendArgs a) {
  if ((int)blockIdx.x < a.weight_blocks * a.R * a.c.heads)  // the longer ones first
    weights<Parts>(a, blockIdx.x);
  else
    join<T, Parts, ONE>(a, blockIdx.x - a.weight_blocks * a.R * a.c.heads);
}

template <class T>
static hipError_t launch_finish(AttendArgs& a, hipStream_t st) {
  const int heads = a.R * a.q_heads, fit = 256 / (a.c.dim / 4), pairs = a.R * a.c.heads;
  const bool parted = a.shared || a.splits > 1, one = heads > 2048;
  const int join_blocks = !parted ? 0 : one ? (heads + fit - 1) / fit : heads;
  // no more workgroups than the card starts in a few microseconds
  a.weight_blocks = a.weight_out ? max(1, min((a.max_len + 1023) / 1024, 4096 / pairs)) : 0;
  const dim3 grid(join_blocks + pairs * a.weight_blocks), threads(256);
  if (grid.x == 0) return hipSuccess;
  if (!parted)
    cache_attend_finish<T, Whole, true><<<grid, threads, 0, st>>>(a);
  else if (a.shared && one)
    cache_attend_finish<T, Shares, true><<<grid, threads, 0, st>>>(a);
  else if (a.shared)
    cache_attend_finish<T, Shares, false><<<grid, threads, 0, st>>>(a);
  else if (one)
    cache_attend_finish<T, Splits, true><<<grid, threads, 0, st>>>(a);
  else
    cache_attend_finish<T, Splits, false><<<grid, threads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_attend_bf16(const AttendArgs& a, hipStream_t st);
hipError_t launch_cache_attend_f32(const AttendArgs& a, hipStream_t st);

hipError_t launch_cache_attend(int bf16, AttendArgs& a, hipStream_t st) {
  const hipError_t e = bf16 ? launch_cache_attend_bf16(a, st) : launch_cache_attend_f32(a, st);
  if (e != hipSuccess) return e;
  return bf16 ? launch_finish<__bf16>(a, st) : launch_finish<float>(a, st);
}

}  // namespace kb
