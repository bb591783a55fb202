// Attention of one new token a row over its cached slots, on the matrix cores.
//
//   x_t = scale * (q . k_t),   out = sum_t e^(x_t - m) v_t / sum_t e^(x_t - m),   m = max x_t
//
// One pass with the running maximum and sum of a softmax: a tile of scores takes (m, s, o) to
// (m', s a + sum e^(x - m'), o a + sum e^(x - m') v), a = e^(m - m').
//
// What bounds it is the cache's stream from memory, 2 dim values a slot and key-value head, which
// every query head that shares the key-value head takes part in.  So a wave holds the queries of 16
// such heads in registers (fewer: zeros) and reads each slot once:
//
//  - S^T = K Q^T in 16 x 16 blocks, rows slots and columns heads.  A lane's part of the operand K is
//    16 bytes of one slot's key, loaded straight from the cache: the sum over the head's values may
//    run in any order, so the lanes of a slot take turns over its 64-byte pieces.
//  - A lane then has the scores of one head for 4 slots of each block, and that is already its part
//    of the operand P^T of the second product, O^T = V^T P^T, if the slots are summed over in that
//    order: probabilities never leave their registers.  o and a have the same head in the lane, so
//    rescaling is a product a register.
//  - A lane's part of V^T would be one value of each of its slots.  It loads 16 bytes of each slot
//    (8 bf16 values; the 16 lanes of a slot read its row from end to end) and picks the value of
//    each product out of them with byte permutations.
//
// bf16: 32 slots a tile, probabilities as two bf16 pieces (the rounding of one alone, 2^-9 of each,
// would double the error of a rounded output; the second product is not what bounds the kernel).
// float32: 16 slots a tile, products on the fp32 matrix instruction.
//
// Kernel time, the least of 20: 128 rows of 8 key-value heads with 4,096 slots of 128 bf16 values 355 us,
// 6.05 TB/s (a large read: 6.06), the matrix cores busy for 6 % of it; one row of 131,072 slots 91 us, and 5 for
// the join; 640 rows of at most 60 slots 13.2 us.
#pragma once

#include "cache_common.hpp"

namespace kb {

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <class T>
struct AttendTile;
template <>
struct AttendTile<__bf16> {
  static constexpr int kSlots = 32;
};
template <>
struct AttendTile<float> {
  static constexpr int kSlots = 16;
};

// The largest (the sum) of the four lanes l, l ^ 16, l ^ 32, l ^ 48, in all of them.
__device__ __forceinline__ float over_groups(float x, bool sum) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  float u = __uint_as_float(a[0]), w = __uint_as_float(a[1]);
  x = sum ? u + w : fmaxf(u, w);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  u = __uint_as_float(b[0]), w = __uint_as_float(b[1]);
  return sum ? u + w : fmaxf(u, w);
}

// What a workgroup of NW waves does with a run of slots [begin, end) of row r for key-value head kv and its
// ht-th 16 query heads.  DC: dim rounded up to a built size.
template <class T, int DC, int NW>
struct AttendRun {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int TS = AttendTile<T>::kSlots, NH = TS / 16;  // slots of a tile, 16-slot blocks
  static constexpr int NI = DC * (int)sizeof(T) / 64;             // 64-byte pieces of a key
  static constexpr int VE = kBf16 && DC > 64 ? 8 : 4;             // values of a slot that a lane holds side by side
  static constexpr int NB = (DC + 16 * VE - 1) / (16 * VE);       // such runs of 16 lanes in a row
  static constexpr int VW = VE * (int)sizeof(T) / 4;              // words of them
  typedef uint32_t Words __attribute__((ext_vector_type(VW)));
  static constexpr int NV = TS / 4;                               // slots of a tile that a lane takes values of
  static constexpr int LD = DC + 4;
  static constexpr int kStep = NW * TS;                           // slots that the waves take at a time

  struct Lds {
    float part[NW > 1 ? NW * 16 * LD : 1];
    float2 stat[NW > 1 ? NW * 16 : 1];
  };

  // The page of this lane's slot of the tile at t0 (any page where the table ends before it).
  static __device__ __forceinline__ int page_of(const AttendArgs& a, const int32_t* pages, int t0) {
    return pages[min(t0 + (int)(threadIdx.x & (TS - 1)), a.max_len - 1) >> a.c.log_ps];
  }

  // page, next_page: page_of the wave's first two tiles.  The results go to `out` and `lse`, or, part_at >=
  // 0, unnormalised to partial part_at + head * part_step.
  static __device__ __forceinline__ void run(const AttendArgs& a, Lds& lds, const int32_t* pages, int r, int kv, int ht,
                                             int begin, int end, int page, int next_page, int64_t part_at,
                                             int part_step) {
    const CacheView& c = a.c;
    const int lane = threadIdx.x & 63, wave = NW > 1 ? threadIdx.x >> 6 : 0;
    const int n = lane & 15, g = lane >> 4;  // operand row or column, group of the summed index
    const int group = a.q_heads / c.heads, h0 = kv * group + ht * 16, nh = min(16, group - ht * 16);
    const int tl = lane & (TS - 1);          // the slot of a tile whose page this lane looks up
    const int first = begin + wave * TS, step = kStep;
    const int D = c.dim, last = D * (int)sizeof(T) / 16 - 1, vlast = D / VE - 1;
    const int row_bytes = D * (int)sizeof(T);

    uint4 q[NI];
    int voff[NB];
    const int g16 = g * 16, last16 = last * 16;  // past the head's end: its last piece again, times zeros
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      q[i] = make_uint4(0, 0, 0, 0);
      if (n < nh && 4 * i + g <= last) {
        const T* p = (const T*)a.q + r * a.q_stride + (int64_t)(h0 + n) * D + (4 * i + g) * (16 / (int)sizeof(T));
        __builtin_memcpy(&q[i], __builtin_assume_aligned(p, sizeof(T)), 16);
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) voff[b] = min(b * 16 + n, vlast) * VW * 4;

    const float scale2 = a.scale * kL2E;
    float m = -FLT_MAX, sum = 0.f;
    f32x4 acc[NB][VE];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < VE; ++e) acc[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};

    if (first < end) {
      uint4 kr[NH][NI];
      Words vr[NV][NB];
      uint32_t valid;
      // this lane's slot as a row of the cache; a hole's or one past the end: some row of the pool
      auto row_at = [&](int page, int t0, uint32_t& ok) {
        const bool there = t0 + tl < end && (uint32_t)page < (uint32_t)c.pages;
        ok = (uint32_t)__ballot(there) & (uint32_t)((1ull << TS) - 1);
        return there ? ((page * c.heads + kv) << c.log_ps) + ((t0 + tl) & ((1 << c.log_ps) - 1)) : 0;
      };
      auto load_k = [&](int row) {
#pragma unroll
        for (int hf = 0; hf < NH; ++hf) {
          const char* p = (const char*)c.k + (int64_t)__shfl(row, hf * 16 + n) * row_bytes;
#pragma unroll
          for (int i = 0; i < NI; ++i) kr[hf][i] = *(const uint4*)(p + min(4 * i * 16 + g16, last16));
        }
      };
      auto load_v = [&](int row) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const char* p = (const char*)c.v + (int64_t)__shfl(row, (j >> 2) * 16 + g * 4 + (j & 3)) * row_bytes;
#pragma unroll
          for (int b = 0; b < NB; ++b) vr[j][b] = *(const Words*)(p + voff[b]);
        }
      };
      int row = row_at(page, first, valid);
      load_k(row);
      load_v(row);

      for (int t0 = first; t0 < end; t0 += step) {
        // scores: x[hf][i] is head n, slot t0 + 16 hf + 4 g + i
        f32x4 x[NH];
#pragma unroll
        for (int hf = 0; hf < NH; ++hf) {
          x[hf] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            if constexpr (kBf16) {
              bf16x8 ka, qb;
              __builtin_memcpy(&ka, &kr[hf][i], 16);
              __builtin_memcpy(&qb, &q[i], 16);
              x[hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qb, x[hf], 0, 0, 0);
            } else {
              float ka[4], qb[4];
              __builtin_memcpy(ka, &kr[hf][i], 16);
              __builtin_memcpy(qb, &q[i], 16);
#pragma unroll
              for (int e = 0; e < 4; ++e) x[hf] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka[e], qb[e], x[hf], 0, 0, 0);
            }
          }
        }
        // The next tile's keys are asked for as soon as this one's registers are free, its values further
        // down: one of the two is always on its way.  Past the last tile they are a row of the pool again:
        // a branch around the loads would have the other half wait for them.  A lone wave has few tiles
        // and is better off without (a call of 640 rows of at most 60 slots, on the device: 14.2 us, 14.8 with
        // them).
        uint32_t next_valid;
        row = row_at(next_page, t0 + step, next_valid);
        next_page = page_of(a, pages, t0 + 2 * step);
        const bool more = NW > 1 || t0 + step < end;
        if (more) load_k(row);

        const bool whole = valid == (uint32_t)((1ull << TS) - 1);
        float top = m;
#pragma unroll
        for (int hf = 0; hf < NH; ++hf)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[hf][i] *= scale2;
            if (!whole && !(valid >> (hf * 16 + g * 4 + i) & 1)) x[hf][i] = -INFINITY;
            top = fmaxf(top, x[hf][i]);
          }
        if (a.scores && n < nh) {
          float* to = a.scores + ((int64_t)r * a.q_heads + h0 + n) * a.score_ld + t0 + g * 4;
#pragma unroll
          for (int hf = 0; hf < NH; ++hf) *(f32x4*)(to + hf * 16) = x[hf];
        }
        top = over_groups(top, false);
        const float keep = exp2_fast(m - top);
        m = top;
        sum *= keep;
#pragma unroll
        for (int hf = 0; hf < NH; ++hf)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[hf][i] = exp2_fast(x[hf][i] - top);
            sum += x[hf][i];
          }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < VE; ++e) acc[b][e] *= keep;

        if (!whole) {  // a probability of 0 times whatever lies there
#pragma unroll
          for (int j = 0; j < NV; ++j) {
            const uint32_t there = 0u - (valid >> ((j >> 2) * 16 + g * 4 + (j & 3)) & 1);
#pragma unroll
            for (int b = 0; b < NB; ++b) vr[j][b] &= there;
          }
        }
        if constexpr (kBf16) {
          bf16x8 hi, lo;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            hi[j] = (__bf16)x[j >> 2][j & 3];
            lo[j] = (__bf16)(x[j >> 2][j & 3] - (float)hi[j]);
          }
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j)
                w[j] = __builtin_amdgcn_perm(vr[2 * j + 1][b][e / 2], vr[2 * j][b][e / 2],
                                             e % 2 ? 0x07060302 : 0x05040100);
              bf16x8 va;
              __builtin_memcpy(&va, w, 16);
              acc[b][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, hi, acc[b][e], 0, 0, 0);
              acc[b][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, lo, acc[b][e], 0, 0, 0);
            }
        } else {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < VE; ++e)
#pragma unroll
              for (int j = 0; j < NV; ++j)
                acc[b][e] =
                    __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[j][b][e]), x[0][j], acc[b][e], 0, 0, 0);
        }
        if (more) load_v(row);
        valid = next_valid;
      }
      sum = over_groups(sum, true);
    }

    // acc[b][e][i]: head n, value (16 b + 4 g + i) VE + e
    auto finish = [&](int head, int d, float* o, float top, float total) {  // 4 values from d
      if (part_at >= 0) {
        const int64_t at = part_at + head * part_step;
        *(f32x4*)(a.part_o + at * D + d) = f32x4{o[0], o[1], o[2], o[3]};
        if (d == 0) a.part_s[at] = make_float2(top, total);
        return;
      }
      const int64_t rh = (int64_t)r * a.q_heads + h0 + head;
      const float norm = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
      T y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = (T)(o[i] * norm);
      __builtin_memcpy(__builtin_assume_aligned((T*)a.out + rh * D + d, 4 * sizeof(T)), y, sizeof y);
      if (d == 0) {
        if (a.lse) a.lse[rh] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * (1.f / kL2E);
        if (a.scores) a.finished[rh] = make_float2(top, norm);
      }
    };
    if constexpr (NW == 1) {
      if (n >= nh) return;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < VE; e += 4) {
            const int d = (16 * b + 4 * g + i) * VE + e;
            float o[4] = {acc[b][e][i], acc[b][e + 1][i], acc[b][e + 2][i], acc[b][e + 3][i]};
            if (d < D) finish(n, d, o, m, sum);
          }
    } else {
      float* part = lds.part;
      float2* stat = lds.stat;
      __syncthreads();  // the run before has been read
      if (g == 0) stat[wave * 16 + n] = make_float2(m, sum);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < VE; e += 4) {
            const int d = (16 * b + 4 * g + i) * VE + e;
            if (n < nh && d < DC)
              *(f32x4*)&part[(wave * 16 + n) * LD + d] =
                  f32x4{acc[b][e][i], acc[b][e + 1][i], acc[b][e + 2][i], acc[b][e + 3][i]};
          }
      __syncthreads();
      for (int i = threadIdx.x; i < nh * (D / 4); i += NW * 64) {
        const int head = i / (D / 4), d = i % (D / 4) * 4;
        float top = -FLT_MAX, total = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, stat[w * 16 + head].x);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const float f = exp2_fast(stat[w * 16 + head].x - top);
          const f32x4 x = *(const f32x4*)&part[(w * 16 + head) * LD + d];
          total += f * stat[w * 16 + head].y;
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] += f * x[j];
        }
        finish(head, d, o, top, total);
      }
    }
  }
};

// A row's splits of a.chunk slots each a workgroup of their own; NW = 1: a wave for a whole row.
template <class T, int DC, int NW>
__global__ __launch_bounds__(NW * 64, DC * sizeof(T) > 256 ? 1 : NW == 1 ? 3 : 2)
void cache_attend_splits(AttendArgs a) {
  using Run = AttendRun<T, DC, NW>;
  __shared__ typename Run::Lds lds;
  const CacheView& c = a.c;
  // All units' first splits, then all second ones: short rows have no later splits, and workgroups go
  // to the XCDs in turn, so the splits of a unit side by side would leave some XCDs without work.
  const int units = a.R * c.heads * a.head_tiles, split = NW == 1 ? 0 : blockIdx.x / units;
  const int unit = blockIdx.x - split * units;
  const int ht = unit % a.head_tiles, kv = unit / a.head_tiles % c.heads, r = unit / a.head_tiles / c.heads;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const int s = cache_seq(c, a.seq, r);
  const int32_t* pages = c.table + (int64_t)max(s, 0) * c.max_pages;
  // The pages of the first two tiles are asked for before the length is known: they, the length and the
  // queries arrive in one round trip.
  const int begin = split * a.chunk, first = begin + (NW > 1 ? threadIdx.x >> 6 : 0) * Run::TS;
  int page = -1, next_page = -1;
  if (a.max_len > 0) page = Run::page_of(a, pages, first), next_page = Run::page_of(a, pages, first + Run::kStep);
  const int len = s < 0 ? 0 : max(0, min(a.length[r], a.max_len)), end = min(len, begin + a.chunk);
  if (a.splits > 1 && begin >= end) return;  // the join knows from the length which splits there are
  if constexpr (NW == 1) {
    Run::run(a, lds, pages, r, kv, ht, 0, len, page, next_page, -1, 0);
  } else {
    const int64_t rh = (int64_t)r * a.q_heads + kv * (a.q_heads / c.heads) + ht * 16;
    Run::run(a, lds, pages, r, kv, ht, begin, end, page, next_page, a.splits > 1 ? rh * a.splits + split : -1,
             a.splits);
  }
}

// Equal shares of all rows' slots: see AttendShares (cache_common.hpp).
template <class T, int DC>
__global__ __launch_bounds__(256, DC * sizeof(T) > 256 ? 1 : 2) void cache_attend_shares(AttendArgs a) {
  using Run = AttendRun<T, DC, 4>;
  __shared__ typename Run::Lds lds;
  __shared__ int pre[kShareRows + 1], len[kShareRows], table_row[kShareRows], wave_sum[4], found;
  const CacheView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, rows = rows_of(a.R, a.n_dev);
  // each XCD a run of neighbouring shares
  const int b = (blockIdx.x & 7) * (kShares / 8) + (blockIdx.x >> 3);

  // The rows' costs in steps, and their sums before each row.
  constexpr int RT = kShareRows / 256;
  int cost[RT], mine = 0;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int r = tid * RT + i;
    cost[i] = 0;
    if (r < rows) {
      const int s = cache_seq(c, a.seq, r), L = s < 0 ? 0 : max(0, min(a.length[r], a.max_len));
      table_row[r] = max(s, 0);
      len[r] = L;
      cost[i] = AttendShares::cost(L, Run::kStep);
    }
    mine += cost[i];
  }
  int before = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int z = __shfl_up(before, d);
    if (lane >= d) before += z;
  }
  if (lane == 63) wave_sum[tid >> 6] = before;
  __syncthreads();
  before -= mine;
  int all = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < tid >> 6) before += wave_sum[w];
    all += wave_sum[w];
  }
  const AttendShares shares(all, c.heads * a.head_tiles);
  const bool idle = b >= shares.shares;
  long long x = idle ? 0 : shares.begin(b);
  const long long x_end = idle ? 0 : shares.begin(b + 1);
  int hp = idle ? 0 : (int)(x / all);
  const int y = (int)(x - (long long)hp * all);  // where in its row's order the first key-value head and 16 heads start
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int r = tid * RT + i;
    if (r <= rows && r < kShareRows) pre[r] = before;
    if (r < rows && before <= y && y < before + cost[i]) found = r;
    if (b == 0 && r < rows) a.row_before[r] = before;  // for the join
    before += cost[i];
    if (r == kShareRows - 1) pre[kShareRows] = before;
  }
  if (b == 0 && tid == 0) a.row_before[rows] = all;
  __syncthreads();

  for (int r = found; x < x_end; ++r) {
    if (r == rows) r = 0, ++hp;
    const long long row_x = (long long)hp * all + pre[r];
    const int o0 = (int)(x - row_x), o1 = (int)(min(x_end, row_x + pre[r + 1] - pre[r]) - row_x);
    x = row_x + o1;
    const bool whole = o0 == 0 && o1 == pre[r + 1] - pre[r];
    const int begin = AttendShares::slot(o0, Run::kStep), end = min(len[r], AttendShares::slot(o1, Run::kStep));
    if (!whole && begin >= end) continue;
    const int kv = hp / a.head_tiles, ht = hp - kv * a.head_tiles;
    const int32_t* pages = c.table + (int64_t)table_row[r] * c.max_pages;
    const int first = begin + (tid >> 6) * Run::TS;
    Run::run(a, lds, pages, r, kv, ht, begin, end, Run::page_of(a, pages, first),
             Run::page_of(a, pages, first + Run::kStep), whole ? -1 : AttendShares::partial(b, o0) * 16, 1);
  }
}

template <class T, int DC>
hipError_t launch_attend_built(const AttendArgs& a, hipStream_t st) {
  const unsigned cells = (unsigned)a.R * a.c.heads * a.head_tiles * a.splits;
  if (a.shared)
    cache_attend_shares<T, DC><<<dim3(kShares), dim3(256), 0, st>>>(a);
  else if (a.waves == 1)
    cache_attend_splits<T, DC, 1><<<dim3(cells), dim3(64), 0, st>>>(a);
  else
    cache_attend_splits<T, DC, 4><<<dim3(cells), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

template <class T>
hipError_t launch_attend_dim(const AttendArgs& a, hipStream_t st) {
  if (a.c.dim <= 64) return launch_attend_built<T, 64>(a, st);
  if (a.c.dim <= 96) return launch_attend_built<T, 96>(a, st);
  if (a.c.dim <= 128) return launch_attend_built<T, 128>(a, st);
  if (a.c.dim <= 192) return launch_attend_built<T, 192>(a, st);
  return launch_attend_built<T, 256>(a, st);
}

}  // namespace kb
