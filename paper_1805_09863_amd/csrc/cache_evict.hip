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
// adding to one address 64 times in turn; the slots kept and those still open are bit masks, 32 slots
// a thread's word, so that the ordered part needs few barriers and later digits are counted of the
// open slots alone.  Lengths above kEvictLds take their keys from memory where these do from LDS.
//
// Kernel time, the least of 20: 16 sequences of 8 heads, 257 slots to 256, 8.4 us; 64 sequences of 8 heads, up to
// 1,100 to 512, 12.7 us; 4 sequences of 8 heads, 32,768 to 2,048, 32 workgroups, 18.5 us (7.6 to read and count
// the first digit, 5.0 for the second, 2.4 for the first masks) and a second launch's 13.1 to move 67 MB in and
// out (5.1 TB/s).  Where choices are compared below, times are whole calls on the device, all launches of them,
// replayed from a graph of ten over two caches in turn.
#include <atomic>

#include "cache_common.hpp"

namespace kb {

constexpr int kEvictLds = 32768;  // keys that fit: 128 KB of LDS, next to 16 KB of counters and 8 KB of masks
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
  // keys, later a list of slots (lengths up to room); two masks, one later a count, for each 32 slots
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

  // Counts of digits; equal digits of a wave: one lane adds.
  auto add = [&](bool in, int digit) {
    const uint64_t ins = __ballot(in);
    if (ins == 0) return;
    if (__popcll(ins) >= 48) {
      const int one = __ffsll((unsigned long long)ins) - 1;
      if (__ballot(in & (digit == __builtin_amdgcn_readlane(digit, one))) == ins) {
        if (lane == one) atomicAdd(&hist[digit * kCopies], __popcll(ins));
        return;
      }
    }
    if (in) atomicAdd(&hist[digit * kCopies + (lane & (kCopies - 1))], 1);
  };
  auto clear = [&] {
    for (int i = tid * 4; i < kDigits * kCopies; i += T * 4) *(int4*)&hist[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
  };
  int need = n, same = L;  // of the `same` slots whose key agrees with T in the bits settled, keep the lowest `need`
  // The digit of T, from the largest down, kDigits / T a thread.
  auto pick_digit = [&] {
    __syncthreads();
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
    need = pick[1], same = pick[2];
    return (uint32_t)pick[0];
  };

  clear();
  if (held && whole) {
    constexpr int U = T / 256;  // 16-byte loads in flight; the last may reach past L, not past the row
    for (int t0 = tid * 4; t0 < L; t0 += U * T * 4) {
      float4 x[U];
      int4 p[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int t = min(t0 + j * T * 4, (L - 1) & ~3);
        x[j] = *(const float4*)(key.weight + t);
        p[j] = key.position ? *(const int4*)(key.position + t) : make_int4(key.lo, key.lo, key.lo, key.lo);
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int t = t0 + j * T * 4;
        if (t >= L) break;
        const uint4 y = make_uint4(key.of(x[j].x, p[j].x), key.of(x[j].y, p[j].y), key.of(x[j].z, p[j].z),
                                   key.of(x[j].w, p[j].w));
        *(uint4*)&lds[t] = y;
        const uint32_t d[4] = {y.x >> 21, y.y >> 21, y.z >> 21, y.w >> 21};
        if (t + 4 <= L) {  // one test for the four: a test each costs more than the counting
          const uint32_t f = __builtin_amdgcn_readfirstlane(d[0]);
          const uint64_t on = __ballot(true);
          if (__ballot(((d[0] ^ f) | (d[1] ^ f) | (d[2] ^ f) | (d[3] ^ f)) == 0) == on) {
            if (lane == __ffsll((unsigned long long)on) - 1) atomicAdd(&hist[f * kCopies], 4 * __popcll(on));
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) atomicAdd(&hist[d[i] * kCopies + (lane & (kCopies - 1))], 1);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 3; ++i)
            if (t + i < L) atomicAdd(&hist[d[i] * kCopies], 1);
        }
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
          add(true, x[j] >> 21);
        }
    }
  }
  uint32_t low_key = pick_digit() << 21, high_key = low_key | ((1u << 21) - 1);  // the keys that agree with T

  const int strips = (L + 63) / 64, words = (L + 31) / 32;
  uint32_t* marks = lds + (held ? room : 0);  // a strip's 2 words of kept slots, 2 of open ones
  auto word = [](int i) { return i / 2 * 4 + (i & 1); };  // word i of the kept slots; its open ones 2 on
  auto key_at = [&](int t) { return held ? lds[t] : key(t); };
  // The slots kept for a key above those that agree with T, and those that agree, the open ones.  With keys in
  // LDS a thread takes a word, its 16-byte pieces in an order that has a wave read from all banks (a strip a
  // wave, by ballots: 12,600 cycles for 512 strips, this 5,000); keys in memory are read in their order.
  auto mark = [&] {
    if (held) {
      for (int i = tid; i < strips * 2; i += T) {
        const int left = L - i * 32;
        const uint32_t in = left >= 32 ? ~0u : left > 0 ? (1u << left) - 1 : 0;
        uint32_t more = 0, least = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int at = ((j + i) & 7) * 4;
          const uint4 x = *(const uint4*)&lds[i * 32 + at];
          auto four = [&](auto f) {
            uint32_t b = f(x.w);
            b = b + b + f(x.z);
            b = b + b + f(x.y);
            return b + b + f(x.x);
          };
          more |= four([&](uint32_t k) { return k > high_key; }) << at;
          least |= four([&](uint32_t k) { return k >= low_key; }) << at;
        }
        marks[word(i)] = more & in, marks[word(i) + 2] = least & ~more & in;
      }
      return;
    }
    for (int s = w; s < strips; s += W) {
      const uint32_t x = key(min(s * 64 + lane, L - 1));
      const uint64_t in = s * 64 + 64 <= L ? ~0ull : (1ull << (L & 63)) - 1;
      const uint64_t more = __ballot(x > high_key) & in, open = __ballot(x >= low_key) & in & ~more;
      if (lane == 0)
        *(uint4*)&marks[s * 4] =
            make_uint4((uint32_t)more, (uint32_t)(more >> 32), (uint32_t)open, (uint32_t)(open >> 32));
    }
  };
  // Where few of many slots are open, the next digits are counted of them alone, a thread a word (32 heads, to
  // 2,048 slots elsewhere, of 32,768: 33.1 us, 39.8 of all slots; with all slots open 54.9 and 45.5; of 16,384:
  // 28.7 and 31.2; of 4,112: 26.3 and 24.8; 128 heads of 257: 12.2 and 9.3).  It takes its bits from the lane's
  // number on, so that the keys that a wave reads lie in many banks.
  const bool few = T == 1024 && L >= 16 * T && same < L / 4;
  const int turn = lane & 31;
  auto open_of = [&](int i) { return __builtin_rotateright32(i < words ? marks[word(i) + 2] : 0, turn); };
  auto slot_of = [&](int i, uint32_t bits) { return i * 32 + ((__ffs(bits) - 1 + turn) & 31); };
  if (few) mark();
  for (int pass = 1; pass < 3 && same != need; ++pass) {
    const int shift = pass == 1 ? 10 : 0, digits = pass == 1 ? 2047 : 1023;
    clear();
    if (few) {
      for (int i = tid; i - tid < words; i += T)
        for (uint32_t bits = open_of(i); __ballot(bits != 0) != 0; bits &= bits - 1)
          add(bits != 0, bits != 0 ? key_at(slot_of(i, bits)) >> shift & digits : 0);
    } else {
#pragma unroll 8
      for (int t = tid; t < L; t += T) {
        const uint32_t x = key_at(t);
        add((x >= low_key) & (x <= high_key), x >> shift & digits);
      }
    }
    low_key |= pick_digit() << shift, high_key = low_key | ((1u << shift) - 1);
    if (few)
      for (int i = tid; i < words; i += T) {
        uint32_t more = 0, open = 0;
        for (uint32_t bits = open_of(i); bits != 0; bits &= bits - 1) {
          const int t = slot_of(i, bits);
          const uint32_t x = key_at(t);
          more |= (uint32_t)(x > high_key) << (t & 31);
          open |= (uint32_t)((x >= low_key) & (x <= high_key)) << (t & 31);
        }
        marks[word(i)] |= more, marks[word(i) + 2] = open;
      }
  }
  if (!few) mark();
  __syncthreads();

  // Open slots are kept, or the lowest `need` of them; each word's kept slots in the words before in the
  // open ones' place.
  int ties = 0, total = 0;
  for (int i0 = 0; i0 < words; i0 += T) {
    const int i = i0 + tid;
    uint32_t open = i < words ? marks[word(i) + 2] : 0;
    int all;
    if (same != need) {
      const int take = max(need - ties - scan<T>(__popc(open), wsum, all), 0);
      ties += all;
      if (take < __popc(open)) {
        uint32_t rest = open;
        for (int j = 0; j < take; ++j) rest &= rest - 1;
        open &= ~rest;
      }
    }
    const uint32_t mine = i < words ? marks[word(i)] | open : 0;
    const int before = total + scan<T>(__popc(mine), wsum, all);
    total += all;
    if (i < words) marks[word(i)] = mine, marks[word(i) + 2] = before;
  }
  __syncthreads();

  // A place t < n of a kept slot is its own; that of a dropped one, the j-th, j = t less the kept ones before
  // it, is the j-th kept slot from n on.
  const int wn = n / 32;
  const uint32_t low = (1u << (n % 32)) - 1;
  const int kept_below = (int)marks[word(wn) + 2] + __popc(marks[word(wn)] & low);
  if (held) {  // those in a list where the keys were
    for (int i = wn + tid; i < words; i += T) {
      uint32_t m = i == wn ? marks[word(i)] & ~low : marks[word(i)];
      for (int j = i == wn ? 0 : (int)marks[word(i) + 2] - kept_below; m != 0; m &= m - 1) lds[j++] = i * 32 + __ffs(m) - 1;
    }
    __syncthreads();
  }
  for (int t0 = w * run; t0 < n; t0 += W * run) {
    const int t = t0 + lane, bit = t & 31;
    const bool live = lane < run && t < n;
    int from = t;
    if (live) {
      const uint32_t m = marks[word(t / 32)];
      const int j = t - (int)marks[word(t / 32) + 2] - __popc(m & ((1u << bit) - 1));
      if (!(m >> bit & 1)) {
        if (held) {
          from = lds[j];
        } else {
          // the last word with at most kept_below + j kept slots before it, then the bit of that rank
          int lo = wn, hi = words;
          while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if ((int)marks[word(mid) + 2] <= kept_below + j) lo = mid; else hi = mid;
          }
          uint32_t bits = marks[word(lo)];
          for (int i = kept_below + j - (int)marks[word(lo) + 2]; i > 0; --i) bits &= bits - 1;
          from = lo * 32 + __ffs(bits) - 1;
        }
      }
      source[t] = from;
    }
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
                          hipFuncAttributeMaxDynamicSharedMemorySize, kEvictLds * 4 + kEvictLds / 64 * 16);
  if (e == hipSuccess) done[dev].store(true, std::memory_order_release);
  return e;
}

template <bool MOVE>
hipError_t launch_select(const EvictArgs& a, hipStream_t st) {
  const int strips = (a.c.cap + 63) / 64, room = min(strips * 64, kEvictLds);
  const size_t lds = max((size_t)room * 4 + room / 64 * 16, (size_t)strips * 16);
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
  // A workgroup moves its head's rows itself where there is one for each CU (512 heads, 4,112 slots to 4,096:
  // 35.7 us, with a second launch 98.4), or for a quarter of them and up to 512 KB of keys and values to move each
  // (64 heads, 8,192 to 7,168: 36.6 and 41.7; 128 heads, 32,768 to 2,048, 1 MB: 88.8 and 82.8), or little to move
  // (128 heads, 257 to 256, 512 bytes: 9.3 and 11.8; 32 heads, 300 to 256, 22 KB: 9.9 and 11.5; 4,112 to 4,096, 8 KB:
  // 16.8 and 18.5); else the whole card does (32 heads, 32,768 to 2,048, 1 MB: 45.2 and 33.1; 4,224 to 4,096, 64 KB:
  // 22.2 and 19.7).
  const int most = a.out_table == a.c.table ? min(places, a.c.cap - places) : places;  // rows of a head that move
  const int64_t bytes = (int64_t)most * a.units * 32, little = a.c.cap <= kEvictSmall ? 128 << 10 : 32 << 10;
  if (pairs >= 256 || bytes <= (pairs >= 64 ? 512 << 10 : little)) {
    const hipError_t e = launch_select<true>(a, st);
    if (e != hipSuccess || a.out_length != a.length) return e;
    cache_evict_lengths<<<(a.R + 255) / 256, 256, 0, st>>>(a);
    return hipGetLastError();
  }
  const hipError_t e = launch_select<false>(a, st);
  if (e != hipSuccess) return e;
  // 16 rows a workgroup at a time, and 16 workgroups a CU (as fast as 8 or 32; with 4 it is 124 us instead of 112
  // for 96 heads, 32,768 slots to 4,096 of 128 values, and 273 instead of 257 for 8 heads, 131,072 to 65,536 of 8)
  const int blocks = min((places + 15) / 16, max(1, 4096 / pairs));
  cache_evict_move<<<dim3(pairs, blocks), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace kb
