// Eviction: a sequence's cache back to its budget, head by head.
//
// Each slot has a 32-bit key (protected slots the largest, then the weights in order, NaN the
// lowest).  One workgroup a sequence and head finds the n-th largest key by a radix selection from
// the top, 11, 11 and 10 bits a pass: T, the bits settled so far of it, and how many of the slots
// that agree with T in them are kept (the lowest ones).  A pass that needs every slot of the digit
// it picks is the last.  The kept slots from n on then fill the places of the dropped slots below
// n; the workgroup moves the rows itself, or a second launch does.
//
// What bounds the selection is the chain of its passes, not the weights' bytes: keys are read once
// and stay in LDS; the two counters a digit keep a wave whose weights share their exponent from
// adding to one address 64 times in turn; kept slots are bit masks, 64 slots each, so that the
// ordered part needs three barriers in all.  Lengths above kEvictLds take their keys from memory in
// every pass.
//
// Kernel time: 16 sequences of 8 heads, 257 slots to 256, 8.4 us (with a second launch 7.4 and 3.1);
// 64 sequences of 8 heads, up to 1,100 to 512, 14.0 us (9 and 7.8); 4 sequences of 8 heads, 32,768 to
// 2,048, 32 workgroups, 28.5 us and a second launch's 13.0 to move 67 MB in and out (5.1 TB/s).
#include <atomic>

#include "cache_common.hpp"

namespace kb {

constexpr int kEvictLds = 32768;  // keys that fit: 128 KB of LDS, next to 16 KB of counters and 6 KB of masks
constexpr int kDigits = 2048, kCopies = 2;

struct EvictKeys {
  const float* weight;
  const int32_t* position;
  int lo, hi;  // protected: positions below lo or above hi
  __device__ __forceinline__ uint32_t of(float w, int p) const {
    w += 0.f;  // -0 counts as 0
    const uint32_t u = __float_as_uint(w);
    const uint32_t key = w == w ? u ^ ((uint32_t)((int)u >> 31) | 0x80000000u) : 0;
    return ((p < lo) | (p > hi)) ? 0xFFFFFFFFu : key;
  }
  __device__ __forceinline__ uint32_t operator()(int t) const { return of(weight[t], position ? position[t] : lo); }
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

// The lanes of m below this one.
__device__ __forceinline__ int lanes_below(uint64_t m) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// A wave's places t of head h of row r (live: t < n), whose rows come from slots `from`: weights, positions,
// and the rows that move, 16 lanes a row, kUnroll times 4 rows in flight.
__device__ __forceinline__ void put_places(const EvictArgs& a, int r, int h, int t, int from, bool live) {
  constexpr int kUnroll = 4;
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 63, units = a.units;
  int at = -1, to = -1;
  if (live) {
    const int64_t rh = (int64_t)r * c.heads + h, in = rh * c.cap + from;
    const int64_t out = rh * ((int64_t)a.out_max_pages << c.log_ps) + t;
    a.out_weight[out] = a.weight[in];
    if (a.position) a.out_position[out] = a.position[in];
    at = cache_row(c, c.table + (int64_t)r * c.max_pages, h, from);
    to = cache_row(c, a.out_table + (int64_t)r * a.out_max_pages, h, t);
  }
  const bool moves = at >= 0 && to >= 0 && at != to;
  const uint64_t m = __ballot(moves);
  const int count = __popcll(m), rank = lanes_below(m), lane_to = (moves ? rank : count + lane - rank) * 4;
  at = __builtin_amdgcn_ds_permute(lane_to, at);  // those that move first
  to = __builtin_amdgcn_ds_permute(lane_to, to);
  typedef uint32_t Piece __attribute__((ext_vector_type(4)));
  Piece *k = (Piece*)c.k, *v = (Piece*)c.v;
  for (int i0 = 0; i0 < count; i0 += 4 * kUnroll)
    for (int u0 = 0; u0 < units; u0 += 16) {  // past the last row or its end: that one again
      const int u = min(u0 + (lane & 15), units - 1);
      Piece x[kUnroll], y[kUnroll];
      int64_t put[kUnroll];
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
        const int i = min(i0 + 4 * j + (lane >> 4), count - 1);
        const int64_t get = (int64_t)__shfl(at, i) * units + u;
        put[j] = (int64_t)__shfl(to, i) * units + u;
        x[j] = k[get], y[j] = v[get];
      }
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) k[put[j]] = x[j], v[put[j]] = y[j];
    }
}

// MOVE: the workgroup moves its rows itself.
template <int T, bool MOVE>
__global__ __launch_bounds__(T) void cache_evict_select(EvictArgs a, int room) {
  // keys, later a list of slots (lengths up to room); a mask and a count for each 64 slots
  extern __shared__ __align__(16) uint32_t lds[];
  __shared__ __align__(16) int hist[kDigits * kCopies];
  __shared__ int wsum[T / 64], pick[3];
  const CacheView& c = a.c;
  const int r = blockIdx.x / c.heads, h = blockIdx.x % c.heads, tid = threadIdx.x, lane = tid & 63;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int L = max(0, min(a.length[r], c.cap)), n = min(L, a.keep);
  int32_t* source = a.source + ((int64_t)r * c.heads + h) * a.keep;
  for (int i = n + tid; i < a.keep; i += T) source[i] = -1;
  if (MOVE && h == 0 && tid == 0 && a.out_length != a.length) a.out_length[r] = n;
  constexpr int W = T / 64;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // places that a wave takes at a time: fewer where their rows would keep few waves busy
  const int run = !MOVE || n >= W * 64 ? 64 : n >= W * 32 ? 32 : 16;
  if (L == n) {
    for (int t0 = w * run; t0 < n; t0 += W * run) {
      const int t = t0 + lane;
      const bool live = lane < run && t < n;
      if (live) source[t] = t;
      if constexpr (MOVE) put_places(a, r, h, t, t, live);
    }
    return;
  }
  const int64_t at = ((int64_t)r * c.heads + h) * c.cap;
  // (first >= 0, so that a bound below every int32 protects the lowest one too)
  const long long old = a.recent > 0 ? (long long)a.newest[r] - a.recent : INT_MAX;
  const EvictKeys key{a.weight + at, a.position ? a.position + at : nullptr, a.first,
                      (int)max(old, (long long)INT_MIN)};
  const bool held = L <= room;  // keys in LDS
  const bool whole = (((uintptr_t)key.weight | (uintptr_t)key.position) & 15) == 0 && c.cap % 4 == 0;

  uint32_t top = 0, mask = 0;
  int need = n, same = L;  // of the `same` slots whose key agrees with top in the bits of mask, keep the lowest `need`
  for (int pass = 0; pass < 3 && same != need; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
    for (int i = tid * 4; i < kDigits * kCopies; i += T * 4) *(int4*)&hist[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
    auto count_in = [&](uint32_t x) {
      const bool in = (x & mask) == top;
      const uint64_t ins = __ballot(in);
      if (ins == 0) return;
      const int digit = x >> shift & ((1 << width) - 1);
      if (__popcll(ins) >= 48) {
        const int one = __ffsll((unsigned long long)ins) - 1;
        if (__ballot(in & (digit == __builtin_amdgcn_readlane(digit, one))) == ins) {  // equal digits: one adds
          if (lane == one) atomicAdd(&hist[digit * kCopies], __popcll(ins));
          return;
        }
      }
      if (in) atomicAdd(&hist[digit * kCopies + (lane & (kCopies - 1))], 1);
    };
    if (held && pass > 0) {
#pragma unroll 8
      for (int t = tid; t < L; t += T) count_in(lds[t]);
    } else if (held && whole) {
      constexpr int U = T / 256;  // 16-byte loads in flight; the last may reach past L, not past the row
      for (int t0 = tid * 4; t0 < L; t0 += U * T * 4) {
        float4 w[U];
        int4 p[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
          const int t = min(t0 + j * T * 4, (L - 1) & ~3);
          w[j] = *(const float4*)(key.weight + t);
          p[j] = key.position ? *(const int4*)(key.position + t) : make_int4(key.lo, key.lo, key.lo, key.lo);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
          const int t = t0 + j * T * 4;
          if (t >= L) break;
          const uint4 x = make_uint4(key.of(w[j].x, p[j].x), key.of(w[j].y, p[j].y), key.of(w[j].z, p[j].z),
                                     key.of(w[j].w, p[j].w));
          *(uint4*)&lds[t] = x;
          count_in(x.x);
          if (t + 1 < L) count_in(x.y);
          if (t + 2 < L) count_in(x.z);
          if (t + 3 < L) count_in(x.w);
        }
      }
    } else {
      constexpr int U = T / 64;  // loads in flight
      for (int t0 = tid; t0 < L; t0 += U * T) {
        uint32_t x[U];
#pragma unroll
        for (int j = 0; j < U; ++j) x[j] = key(min(t0 + j * T, L - 1));
#pragma unroll
        for (int j = 0; j < U; ++j)
          if (t0 + j * T < L) {
            if (held) lds[t0 + j * T] = x[j];
            count_in(x[j]);
          }
      }
    }
    __syncthreads();
    // digits from the largest down, kDigits / T a thread
    constexpr int B = kDigits / T;
    const int d0 = kDigits - 1 - tid * B;
    int copy[B * kCopies], count[B], mine = 0, all;
    __builtin_memcpy(copy, __builtin_assume_aligned(&hist[(d0 - B + 1) * kCopies], 16), sizeof copy);
#pragma unroll
    for (int j = 0; j < B; ++j) {
      count[j] = copy[(B - 1 - j) * kCopies] + copy[(B - 1 - j) * kCopies + 1];
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

  // Each wave takes a run of whole 64-slot strips; what is uniform in it stays on the scalar unit.
  const int strips = (L + 63) / 64;
  const int per = (strips + W - 1) / W, s0 = min(w * per, strips), s1 = min(s0 + per, strips);
  const int marks = held ? room / 64 : strips;
  uint64_t* kept = (uint64_t*)(lds + (held ? room : 0));  // each strip's kept slots
  int* before = (int*)(kept + marks);                     // and their number in the strips before
  auto key_at = [&](int t) { return (held ? lds[min(t, L - 1)] : key(min(t, L - 1))) & mask; };

  int all, ties = 0;  // slots that agree with top, in the strips before
  if (same != need) {
#pragma unroll 4
    for (int s = s0; s < s1; ++s) ties += __popcll(__ballot((s * 64 + lane < L) & (key_at(s * 64 + lane) == top)));
    ties = __builtin_amdgcn_readfirstlane(scan<T>(lane == 0 ? ties : 0, wsum, all));
  }
  int count = 0;  // of the wave's kept slots
  uint64_t mine = 0;
  for (int batch = s0; batch < s1; batch += 64) {  // lane j: strip batch + j; with keys in LDS there is one batch
    mine = 0;
#pragma unroll 4
    for (int s = batch; s < min(s1, batch + 64); ++s) {
      const int t = s * 64 + lane;
      const uint32_t x = key_at(t);
      uint64_t m;
      if (same == need) {
        m = __ballot((t < L) & (x >= top));
      } else {
        const uint64_t tie = __ballot((t < L) & (x == top));
        m = __ballot((t < L) & ((x > top) | ((x == top) & (ties + lanes_below(tie) < need))));
        ties += __popcll(tie);
      }
      mine = lane == s - batch ? m : mine;
    }
    int sum = __popcll(mine);
    const int own = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int z = __shfl_up(sum, d);
      if (lane >= d) sum += z;
    }
    if (batch + lane < s1) kept[batch + lane] = mine, before[batch + lane] = count + sum - own;
    count += __shfl(sum, 63);
  }
  // scan<T>'s barriers also part the keys' last reads from the list that takes their place
  count = scan<T>(lane == 0 ? count : 0, wsum, all);
  count = __shfl(count, 0);
  for (int s = s0 + lane; s < s1; s += 64) before[s] += count;
  __syncthreads();

  // A place t < n of a kept slot is its own; that of a dropped one, the j-th, j = t less the kept ones before
  // it, is the j-th kept slot from n on.
  const int sn = n / 64;
  const uint64_t low = (1ull << (n % 64)) - 1;
  const int kept_below = before[sn] + __popcll(kept[sn] & low);
  if (held) {
    // Those in a list where the keys were: a slot's rank among the kept ones less that of slot n.  (32 strips a
    // wave: a lane a strip, bit by bit, 2,100 cycles at 1 slot in 16 kept against 9,500 strip by strip; 8
    // strips a wave: strip by strip, 1,800 against 3,300.)
    const int s = s0 + lane, rank = s < s1 ? before[s] - kept_below : 0;
    if constexpr (T == 1024) {
      if (s >= sn && s < s1) {
        uint64_t m = s == sn ? mine & ~low : mine;
        for (int i = s == sn ? 0 : rank; m != 0; m &= m - 1)
          lds[i++] = s * 64 + __ffsll((unsigned long long)m) - 1;
      }
    } else {
      for (int z = max(s0, sn); z < s1; ++z) {
        uint64_t m = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)mine, z - s0) |
                     (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), z - s0) << 32;
        const int first = z == sn ? 0 : __builtin_amdgcn_readlane(rank, z - s0);
        if (z == sn) m &= ~low;
        if (__builtin_amdgcn_inverse_ballot_w64(m)) lds[first + lanes_below(m)] = z * 64 + lane;
      }
    }
    __syncthreads();
  }
  for (int t0 = w * run; t0 < n; t0 += W * run) {
    const int t = t0 + lane, s = t0 / 64, bit = t & 63;
    const uint64_t m = kept[s];
    const bool live = lane < run && t < n, stays = m >> bit & 1;
    const int j = t - before[s] - __popcll(m & ((1ull << bit) - 1));
    int from = t;
    if (live && !stays) {
      if (held) {
        from = lds[j];
      } else {
        // the last strip with at most kept_below + j kept slots before it, then the bit of that rank
        int lo = sn, hi = strips;
        while (hi - lo > 1) {
          const int mid = (lo + hi) / 2;
          if (before[mid] <= kept_below + j) lo = mid; else hi = mid;
        }
        uint64_t bits = kept[lo];
        for (int i = kept_below + j - before[lo]; i > 0; --i) bits &= bits - 1;
        from = lo * 64 + __ffsll((unsigned long long)bits) - 1;
      }
    }
    if (live) source[t] = from;
    if constexpr (MOVE) put_places(a, r, h, t, from, live);
  }
}

__device__ __forceinline__ int kept_of(const EvictArgs& a, int r) {
  return min(max(0, min(a.length[r], a.c.cap)), a.keep);
}

// Rows to their places by the whole card: 16 lanes a row, 16 bytes of key and value each at a time.
__global__ __launch_bounds__(256) void cache_evict_move(EvictArgs a) {
  const CacheView& c = a.c;
  const int units = a.units;
  const int r = blockIdx.x / c.heads, h = blockIdx.x % c.heads, lane = threadIdx.x % 16;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int places = min(a.keep, c.cap);
  const int64_t rh = (int64_t)r * c.heads + h;
  const int32_t *source = a.source + rh * a.keep, *from_t = c.table + (int64_t)r * c.max_pages,
                *to_t = a.out_table + (int64_t)r * a.out_max_pages;
  const int64_t in = rh * c.cap, out = rh * ((int64_t)a.out_max_pages << c.log_ps);
  const uint4 *k = (const uint4*)c.k, *v = (const uint4*)c.v;
  for (int i = blockIdx.y * 16 + threadIdx.x / 16; i < places; i += gridDim.y * 16) {
    const int s = source[i], to = cache_row(c, to_t, h, i);
    if (s < 0) break;
    const int from = cache_row(c, from_t, h, s);
    if (from >= 0 && to >= 0 && from != to)
      for (int u = lane; u < units; u += 16) {
        const uint4 x = k[(int64_t)from * units + u], y = v[(int64_t)from * units + u];
        ((uint4*)c.k)[(int64_t)to * units + u] = x;
        ((uint4*)c.v)[(int64_t)to * units + u] = y;
      }
    if (lane == 0) {
      a.out_weight[out + i] = a.weight[in + s];
      if (a.position) a.out_position[out + i] = a.position[in + s];
    }
  }
  if (h == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.out_length[r] = kept_of(a, r);
}

// New lengths in place of the old ones, which every head's workgroup above reads.
__global__ __launch_bounds__(256) void cache_evict_lengths(EvictArgs a) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r < rows_of(a.R, a.n_dev)) a.out_length[r] = kept_of(a, r);
}

// A workgroup of 256 threads holds up to 2,048 keys: its passes are shorter than those of 1,024
// threads, and more workgroups share a unit.
constexpr int kEvictSmall = 2048;

// Raises the long kernel's LDS ceiling, once per device.
template <bool MOVE>
hipError_t raise_lds_ceiling() {
  constexpr int kMaxDevices = 64;
  static std::atomic<bool> done[kMaxDevices];
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess || dev < 0 || dev >= kMaxDevices) return e != hipSuccess ? e : hipErrorInvalidDevice;
  if (done[dev].load(std::memory_order_acquire)) return hipSuccess;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(&cache_evict_select<1024, MOVE>),
                          hipFuncAttributeMaxDynamicSharedMemorySize, kEvictLds * 4 + kEvictLds / 64 * 12);
  if (e == hipSuccess) done[dev].store(true, std::memory_order_release);
  return e;
}

template <bool MOVE>
hipError_t launch_select(const EvictArgs& a, hipStream_t st) {
  const int strips = (a.c.cap + 63) / 64, room = min(strips * 64, kEvictLds);
  const size_t lds = max((size_t)room * 4 + room / 64 * 12, (size_t)strips * 12);
  const dim3 grid(a.R * a.c.heads);
  if (room <= kEvictSmall) {
    cache_evict_select<256, MOVE><<<grid, dim3(256), lds, st>>>(a, room);
  } else {
    const hipError_t e = raise_lds_ceiling<MOVE>();
    if (e != hipSuccess) return e;
    cache_evict_select<1024, MOVE><<<grid, dim3(1024), lds, st>>>(a, room);
  }
  return hipGetLastError();
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t st) {
  const int pairs = a.R * a.c.heads, places = min(a.keep, a.c.cap);
  // A workgroup moves its head's rows itself where there are workgroups for half the card (512 heads, 4,112
  // slots to 4,096: 36 us, with a second launch 97; 128 heads, 2,000 to 1,500: 25 and 27), or it has little to
  // move (32 heads of 300 slots to 256 elsewhere, 128 KB: 10.0 and 11.0; of 4,112 to 4,096, 8 KB: 16.9 and
  // 18.7), else the whole card does (32 heads, 32,768 slots to 2,048, 1 MB: 40 us, by the workgroups 53; of
  // 4,352 to 4,096, 128 KB: 22.7 and 25.4).
  const int most = a.out_table == a.c.table ? min(places, a.c.cap - places) : places;  // rows of a head that move
  const int64_t few = a.c.cap <= kEvictSmall ? 128 << 10 : 32 << 10;
  if (pairs >= 128 || (int64_t)most * a.units * 32 <= few) {
    const hipError_t e = launch_select<true>(a, st);
    if (e != hipSuccess || a.out_length != a.length) return e;
    cache_evict_lengths<<<(a.R + 255) / 256, 256, 0, st>>>(a);
    return hipGetLastError();
  }
  const hipError_t e = launch_select<false>(a, st);
  if (e != hipSuccess) return e;
  // 16 rows a workgroup at a time, and 16 workgroups a CU (rows of 128 values: as fast as 8 or 32, with 4 it is
  // 131 us instead of 119 for 96 heads, 32,768 slots to 4,096; 8 heads, 131,072 to 65,536, rows of 8 values:
  // 282 us, with 8 a CU 318)
  const int blocks = min((places + 15) / 16, max(1, 4096 / pairs));
  cache_evict_move<<<dim3(pairs, blocks), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace kb
