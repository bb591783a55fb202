// Eviction: a sequence's cache back to its budget, head by head.
//
// Each slot has a 32-bit key (protected slots the largest, then the weights in
// order, NaN the lowest).  A radix selection, 8 bits a pass, finds the n-th
// largest key T and how many of the slots with exactly that key are kept (the
// lowest ones).  The kept slots from n on then fill the places of the dropped
// slots below n.
#include "cache_common.hpp"

namespace kb {

constexpr int kEvictT = 1024;

struct EvictKeys {
  const float* weight;
  const int32_t* position;
  int first, recent, newest;
  __device__ __forceinline__ uint32_t operator()(int t) const {
    if (position) {
      const int p = position[t];
      if (p < first || (recent > 0 && (long long)p > (long long)newest - recent)) return 0xFFFFFFFFu;
    }
    const float w = weight[t] + 0.f;  // -0 counts as 0
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  }
};

// Exclusive prefix sums over the workgroup; total: the whole sum.
__device__ __forceinline__ int scan(int x, int* wave_sums, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int y = x;
  for (int d = 1; d < 64; d <<= 1) {
    const int z = __shfl_up(y, d);
    if (lane >= d) y += z;
  }
  if (lane == 63) wave_sums[w] = y;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int i = 0; i < kEvictT / 64; ++i) {
    if (i < w) before += wave_sums[i];
    total += wave_sums[i];
  }
  __syncthreads();
  return before + y - x;
}

__global__ __launch_bounds__(kEvictT) void cache_evict_select(EvictArgs a) {
  __shared__ int hist[256], wsum[kEvictT / 64], pick, rest;
  const CacheView& c = a.c;
  const int r = blockIdx.x / c.heads, h = blockIdx.x % c.heads, tid = threadIdx.x;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int L = max(0, min(a.length[r], c.cap)), n = min(L, a.keep);
  int32_t* source = a.source + ((int64_t)r * c.heads + h) * a.keep;
  for (int i = n + tid; i < a.keep; i += kEvictT) source[i] = -1;
  if (L == n) {
    for (int i = tid; i < n; i += kEvictT) source[i] = i;
    return;
  }
  const int64_t at = ((int64_t)r * c.heads + h) * c.cap;
  const EvictKeys key{a.weight + at, a.position ? a.position + at : nullptr, a.first, a.recent,
                      a.newest ? a.newest[r] : 0};

  uint32_t T = 0, mask = 0;
  int need = n;  // of the slots whose key agrees with T in the bits of mask
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int t = tid; t < L; t += kEvictT) {
      const uint32_t x = key(t);
      if ((x & mask) == T) atomicAdd(&hist[(x >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int b = 255, left = need;
      while (hist[b] < left) left -= hist[b--];
      pick = b;
      rest = left;
    }
    __syncthreads();
    T |= (uint32_t)pick << shift;
    mask |= 255u << shift;
    need = rest;
    __syncthreads();
  }

  // The kept slots from n on, ascending, to the front of source; and the
  // number of ties below n.
  int ties = 0, ties_below = 0, moved = 0, all;
  for (int t0 = 0; t0 < L; t0 += kEvictT) {
    const int t = t0 + tid;
    const uint32_t x = t < L ? key(t) : 0;
    const bool tie = t < L && x == T;
    const int rank = ties + scan(tie, wsum, all);
    ties += all;
    scan(tie && t < n, wsum, all);
    ties_below += all;
    const bool move = t >= n && t < L && (x > T || (tie && rank < need));
    const int to = moved + scan(move, wsum, all);
    if (move) source[to] = t;
    moved += all;
  }
  __syncthreads();
  // Places n - 1 .. 0: a kept slot's own number, a dropped one's the tail slot
  // of its rank.  The j-th dropped place is at j or above, so in descending
  // order no entry of the list is overwritten before it is read.
  int above = 0, ties_above = 0;
  for (int e = n; e > 0; e -= kEvictT) {
    const int t = e - 1 - tid;
    const uint32_t x = t >= 0 ? key(t) : 0;
    const bool tie = t >= 0 && x == T;
    const int tr = ties_below - 1 - (ties_above + scan(tie, wsum, all));
    ties_above += all;
    const bool drop = t >= 0 && !(x > T || (tie && tr < need));
    const int j = moved - 1 - (above + scan(drop, wsum, all));
    above += all;
    const int s = drop ? source[j] : t;
    __syncthreads();
    if (t >= 0) source[t] = s;
    __syncthreads();
  }
}

template <class V>
__global__ __launch_bounds__(256) void cache_evict_move(EvictArgs a, int units) {
  const CacheView& c = a.c;
  const int r = blockIdx.x / c.heads, h = blockIdx.x % c.heads;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int64_t rh = (int64_t)r * c.heads + h;
  const int32_t *source = a.source + rh * a.keep, *from_t = c.table + (int64_t)r * c.max_pages,
                *to_t = a.out_table + (int64_t)r * a.out_max_pages;
  const int64_t in = rh * c.cap, out = rh * ((int64_t)a.out_max_pages << c.log_ps);
  for (int i = blockIdx.y * 16 + threadIdx.x / 16; i < a.keep; i += gridDim.y * 16) {
    const int s = source[i];
    if (s < 0) break;
    const int from = cache_row(c, from_t, h, s), to = cache_row(c, to_t, h, i);
    if (from >= 0 && to >= 0 && from != to)
      for (int u = threadIdx.x % 16; u < units; u += 16) {
        ((V*)c.k)[(int64_t)to * units + u] = ((const V*)c.k)[(int64_t)from * units + u];
        ((V*)c.v)[(int64_t)to * units + u] = ((const V*)c.v)[(int64_t)from * units + u];
      }
    if (threadIdx.x % 16 == 0) {
      a.out_weight[out + i] = a.weight[in + s];
      if (a.position) a.out_position[out + i] = a.position[in + s];
    }
  }
  if (h == 0 && blockIdx.y == 0 && threadIdx.x == 0)
    a.out_length[r] = min(max(0, min(a.length[r], c.cap)), a.keep);
}

hipError_t launch_cache_evict(int bf16, const EvictArgs& a, hipStream_t st) {
  cache_evict_select<<<dim3(a.R * a.c.heads), dim3(kEvictT), 0, st>>>(a);
  const int blocks = min(1024, (a.keep + 63) / 64);
  cache_evict_move<uint4><<<dim3(a.R * a.c.heads, blocks), dim3(256), 0, st>>>(a, a.c.dim * (bf16 ? 2 : 4) / 16);
  return hipGetLastError();
}

}  // namespace kb
