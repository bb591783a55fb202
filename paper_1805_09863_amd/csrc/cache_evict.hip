// Eviction: a sequence's cache back to its budget, head by head.
//
// Each slot has a 32-bit key (protected slots the largest, then the weights in order, NaN the
// lowest).  One workgroup a sequence and head finds the n-th largest key by a radix selection from
// the top, 11, 11 and 10 bits a pass: T, the bits settled so far of it, and how many of the slots
// that agree with T in them are kept (the lowest ones).  A pass that needs every slot of the digit
// it picks is the last.  The kept slots from n on then fill the places of the dropped slots below
// n, and a second kernel moves the rows.
//
// What bounds the selection is the chain of its passes, not the weights' bytes: keys are read once
// and stay in LDS; the two counters a digit keep a wave whose weights share their exponent from
// adding to one address 64 times in turn; kept slots are bit masks, 64 slots each, so that the
// ordered part needs three barriers in all.  Lengths above kEvictLds take their keys from memory in
// every pass and go through the ordered part 1,024 slots at a time.
#include <atomic>

#include "cache_common.hpp"

namespace kb {

constexpr int kEvictLds = 32768;  // keys that fit: 128 KB of LDS, next to 16 KB of counters
constexpr int kDigits = 2048, kCopies = 2;

struct EvictKeys {
  const float* weight;
  const int32_t* position;
  int first, recent, newest;
  __device__ __forceinline__ uint32_t operator()(int t) const {
    const float w = weight[t] + 0.f;  // -0 counts as 0
    const uint32_t u = __float_as_uint(w);
    uint32_t key = w != w ? 0 : (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    if (position) {
      const int p = position[t];
      if (p < first || (recent > 0 && (long long)p > (long long)newest - recent)) key = 0xFFFFFFFFu;
    }
    return key;
  }
};

// Exclusive prefix sums over the workgroup; total: the whole sum.
template <int T>
__device__ __forceinline__ int scan(int x, int* wave_sums, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int y = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int z = __shfl_up(y, d);
    if (lane >= d) y += z;
  }
  if (lane == 63) wave_sums[w] = y;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < T / 64; ++i) {
    const int z = wave_sums[i];
    if (i < w) before += z;
    total += z;
  }
  __syncthreads();
  return before + y - x;
}

template <int T>
__global__ __launch_bounds__(T) void cache_evict_select(EvictArgs a, int room) {
  extern __shared__ uint32_t lds[];  // room keys, later a list of tail slots; room / 64 masks of kept slots
  __shared__ __align__(16) int hist[kDigits * kCopies];
  __shared__ int wsum[T / 64], wsum2[T / 64], pick[3];
  const CacheView& c = a.c;
  const int r = blockIdx.x / c.heads, h = blockIdx.x % c.heads, tid = threadIdx.x;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int L = max(0, min(a.length[r], c.cap)), n = min(L, a.keep);
  int32_t* source = a.source + ((int64_t)r * c.heads + h) * a.keep;
  for (int i = n + tid; i < a.keep; i += T) source[i] = -1;
  if (L == n) {
    for (int i = tid; i < n; i += T) source[i] = i;
    return;
  }
  const int64_t at = ((int64_t)r * c.heads + h) * c.cap;
  const EvictKeys key{a.weight + at, a.position ? a.position + at : nullptr, a.first, a.recent,
                      a.newest ? a.newest[r] : 0};
  const bool held = L <= room;  // keys in LDS

  uint32_t top = 0, mask = 0;
  int need = n, same = L;  // of the `same` slots whose key agrees with top in the bits of mask, keep the lowest `need`
  for (int pass = 0; pass < 3 && same != need; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
    for (int i = tid * 4; i < kDigits * kCopies; i += T * 4) *(int4*)&hist[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
    for (int t = tid; t < L; t += T) {
      const uint32_t x = held && pass > 0 ? lds[t] : key(t);
      if (held && pass == 0) lds[t] = x;
      if ((x & mask) == top) atomicAdd(&hist[(x >> shift & ((1u << width) - 1)) * kCopies + (tid & (kCopies - 1))], 1);
    }
    __syncthreads();
    // digits from the largest down, kDigits / T a thread
    constexpr int B = kDigits / T;
    const int d0 = kDigits - 1 - tid * B;
    int count[B], mine = 0, all;
#pragma unroll
    for (int j = 0; j < B; ++j) {
      count[j] = hist[(d0 - j) * kCopies] + hist[(d0 - j) * kCopies + 1];
      mine += count[j];
    }
    int before = scan<T>(mine, wsum, all);
#pragma unroll
    for (int j = 0; j < B; ++j) {
      if (before < need && need <= before + count[j]) pick[0] = d0 - j, pick[1] = need - before, pick[2] = count[j];
      before += count[j];
    }
    __syncthreads();
    top |= (uint32_t)pick[0] << shift;
    mask |= ((1u << width) - 1) << shift;
    need = pick[1], same = pick[2];
  }

  if (held) {
    // Each wave: a run of whole 64-slot strips.
    constexpr int W = T / 64;
    const int lane = tid & 63, w = tid >> 6, strips = (L + 63) / 64;
    const int s0 = (int)((long long)strips * w / W), s1 = (int)((long long)strips * (w + 1) / W);
    uint64_t* kept = (uint64_t*)(lds + room);
    const uint64_t below = (1ull << lane) - 1;
    int ties = 0;  // slots that agree with top, in the strips before
    if (same != need) {
      for (int s = s0; s < s1; ++s) ties += __popcll(__ballot(s * 64 + lane < L && (lds[s * 64 + lane] & mask) == top));
      int all;
      const int before = scan<T>(lane == 0 ? ties : 0, wsum, all);
      ties = __shfl(before, 0);
    }
    int tail = 0, holes = 0;  // kept slots from n on, dropped ones below n
    for (int s = s0; s < s1; ++s) {
      const int t = s * 64 + lane;
      const uint32_t x = t < L ? lds[t] & mask : 0;
      const uint64_t tie = __ballot(t < L && x == top);
      const bool stay = t < L && (x > top || (x == top && ties + __popcll(tie & below) < need));
      ties += __popcll(tie);
      const uint64_t m = __ballot(stay);
      if (lane == 0) kept[s] = m;
      tail += __popcll(__ballot(stay && t >= n));
      holes += __popcll(__ballot(!stay && t < n));
    }
    if (lane == 0) wsum[w] = tail, wsum2[w] = holes;
    __syncthreads();
    tail = holes = 0;
    for (int i = 0; i < w; ++i) tail += wsum[i], holes += wsum2[i];
    // the keys have been read: their place is the list's
    for (int s = max(s0, n / 64); s < s1; ++s) {
      const int t = s * 64 + lane;
      const uint64_t from_n = s * 64 >= n ? ~0ull : ~0ull << (n - s * 64), m = kept[s] & from_n;
      if (m >> lane & 1) lds[tail + __popcll(m & below)] = t;
      tail += __popcll(m);
    }
    __syncthreads();
    for (int s = s0; s < s1 && s * 64 < n; ++s) {
      const int t = s * 64 + lane;
      const uint64_t m = ~kept[s];  // ones at and after n belong to no place
      if (t < n) source[t] = (m >> lane & 1) ? (int)lds[holes + __popcll(m & below)] : t;
      holes += __popcll(m);
    }
    return;
  }

  // The kept slots from n on, ascending, to the front of source; and the number of ties below n.
  int ties = 0, ties_below = 0, moved = 0, all;
  for (int t0 = 0; t0 < L; t0 += T) {
    const int t = t0 + tid;
    const uint32_t x = t < L ? key(t) & mask : 0;
    const bool tie = t < L && x == top;
    const int rank = ties + scan<T>(tie, wsum, all);
    ties += all;
    scan<T>(tie && t < n, wsum, all);
    ties_below += all;
    const bool move = t >= n && t < L && (x > top || (tie && rank < need));
    const int to = moved + scan<T>(move, wsum, all);
    if (move) source[to] = t;
    moved += all;
  }
  __syncthreads();
  // Places n - 1 .. 0: a kept slot's own number, a dropped one's the tail slot of its rank.  The
  // j-th dropped place is at j or above, so in descending order no entry of the list is
  // overwritten before it is read.
  int above = 0, ties_above = 0;
  for (int e = n; e > 0; e -= T) {
    const int t = e - 1 - tid;
    const uint32_t x = t >= 0 ? key(t) & mask : 0;
    const bool tie = t >= 0 && x == top;
    const int tr = ties_below - 1 - (ties_above + scan<T>(tie, wsum, all));
    ties_above += all;
    const bool drop = t >= 0 && !(x > top || (tie && tr < need));
    const int j = moved - 1 - (above + scan<T>(drop, wsum, all));
    above += all;
    const int s = drop ? source[j] : t;
    __syncthreads();
    if (t >= 0) source[t] = s;
    __syncthreads();
  }
}

// Rows to their places: 16 lanes a row, 16 bytes of key and value each at a time.
__global__ __launch_bounds__(256) void cache_evict_move(EvictArgs a, int units) {
  const CacheView& c = a.c;
  const int r = blockIdx.x / c.heads, h = blockIdx.x % c.heads;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int n = min(max(0, min(a.length[r], c.cap)), a.keep);
  const int64_t rh = (int64_t)r * c.heads + h;
  const int32_t *source = a.source + rh * a.keep, *from_t = c.table + (int64_t)r * c.max_pages,
                *to_t = a.out_table + (int64_t)r * a.out_max_pages;
  const int64_t in = rh * c.cap, out = rh * ((int64_t)a.out_max_pages << c.log_ps);
  const uint4 *k = (const uint4*)c.k, *v = (const uint4*)c.v;
  for (int i = blockIdx.y * 16 + threadIdx.x / 16; i < n; i += gridDim.y * 16) {
    const int s = source[i];
    const int from = cache_row(c, from_t, h, s), to = cache_row(c, to_t, h, i);
    if (from >= 0 && to >= 0 && from != to)
      for (int u = threadIdx.x % 16; u < units; u += 16) {
        const uint4 x = k[(int64_t)from * units + u], y = v[(int64_t)from * units + u];
        ((uint4*)c.k)[(int64_t)to * units + u] = x;
        ((uint4*)c.v)[(int64_t)to * units + u] = y;
      }
    if (threadIdx.x % 16 == 0) {
      a.out_weight[out + i] = a.weight[in + s];
      if (a.position) a.out_position[out + i] = a.position[in + s];
    }
  }
  if (h == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.out_length[r] = n;
}

// A workgroup of 256 threads holds up to 2,048 keys: its passes are shorter than those of 1,024
// threads, and more workgroups share a unit.
constexpr int kEvictSmall = 2048;

// Raises the kernel's LDS ceiling, once per device.
static hipError_t raise_lds_ceiling() {
  constexpr int kMaxDevices = 64;
  static std::atomic<bool> done[kMaxDevices];
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess || dev < 0 || dev >= kMaxDevices) return e != hipSuccess ? e : hipErrorInvalidDevice;
  if (done[dev].load(std::memory_order_acquire)) return hipSuccess;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(&cache_evict_select<1024>),
                          hipFuncAttributeMaxDynamicSharedMemorySize, kEvictLds * 4 + kEvictLds / 8);
  if (e == hipSuccess) done[dev].store(true, std::memory_order_release);
  return e;
}

hipError_t launch_cache_evict(int bf16, const EvictArgs& a, hipStream_t st) {
  const int room = min((a.c.cap + 63) / 64 * 64, kEvictLds);
  const size_t lds = (size_t)room * 4 + room / 8;
  const dim3 grid(a.R * a.c.heads);
  if (room <= kEvictSmall) {
    cache_evict_select<256><<<grid, dim3(256), lds, st>>>(a, room);
  } else {
    const hipError_t e = raise_lds_ceiling();
    if (e != hipSuccess) return e;
    cache_evict_select<1024><<<grid, dim3(1024), lds, st>>>(a, room);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int blocks = min(1024, (min(a.keep, a.c.cap) + 63) / 64);
  cache_evict_move<<<dim3(a.R * a.c.heads, blocks), dim3(256), 0, st>>>(a, a.c.dim * (bf16 ? 2 : 4) / 16);
  return hipGetLastError();
}

}  // namespace kb
