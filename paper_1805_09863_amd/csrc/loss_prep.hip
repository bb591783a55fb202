// Around the products of the output layer's losses: which rows count and their entries, operands laid out for the
// DMA pipeline, and the losses from the parts of all splits.
#include <algorithm>

#include "k3_scan.hpp"
#include "loss_bias.hpp"
#include "loss_common.hpp"
#include "loss_load.hpp"
#include "loss_teacher.hpp"

namespace kb {

typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));

// Teachers' rows, a wave each.
__global__ __launch_bounds__(256) void loss_teacher(LossTeacherArgs a) {
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.N) return;
  const TeacherRow r = teacher_row(a.token + (size_t)row * a.K, a.logit + (size_t)row * a.K, a.K, a.V, a.inv_t);
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (lane + 64 * u < a.K) {
      const size_t at = (size_t)row * a.K + lane + 64 * u;
      a.out_token[at] = r.token[u];
      a.part[at] = r.part[u];
    }
  if (lane == 0) {
    a.known[row] = r.known;
    a.flag[row] = r.any;
  }
}

__device__ __forceinline__ bool row_counts(const LossRows& a, int n) {
  if (a.flag) return a.flag[n] != 0;
  const int t = a.token[n];
  return t >= 0 && t < a.V;
}

// Rows that count, in order (a stable compaction).  One workgroup: 4,096 rows a turn.
__global__ __launch_bounds__(K3_T) void loss_rows(LossRows a) {
  __shared__ int wsum[K3_W];
  for (int n = threadIdx.x; n < a.N; n += K3_T)
    if (!row_counts(a, n)) a.inv[n] = -1;
  const int kept = compact_entries_pass(
      a.N, [&](int n) { return row_counts(a, n); },
      [&](int c, int n) {
        a.map[c] = n;
        a.inv[n] = c;
      },
      wsum);
  if (threadIdx.x == 0) *a.count = kept;
}

// x in `planes` bf16 pieces.
template <int PLANES>
__device__ __forceinline__ void write_pieces(const float (&x)[8], uint16_t* out, size_t plane) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
  for (int p = 0; p < PLANES; ++p) {
    bf16x8v v;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = (__bf16)r[i];
      r[i] -= (float)v[i];
    }
    *reinterpret_cast<bf16x8v*>(out + p * plane) = v;
  }
}

// n of 8 values from p on, the rest zeros; all of them by loads of 16 bytes, at any address.
template <class S>
__device__ __forceinline__ void load8(const S* p, int n, float (&x)[8]) {
  if (n >= 8) {
    load16(p, x);
    if constexpr (sizeof(S) == 4) load16(p + 4, x + 4);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = i < n ? widen(p, i) : 0.f;
}

template <class S, int PLANES>
__device__ __forceinline__ void pack_w(const LossPackWArgs& a, long long first, long long step) {
  const int chunks = a.Vc / 8;
  const long long total = (long long)a.Hk * chunks;
  for (long long i = first; i < total; i += step) {
    const int r = (int)(i / chunks), w = (int)(i % chunks) * 8;
    float x[8];
    const int n = a.V - a.v0 - w;
    if (r < a.H && n > 0) {
      load8(static_cast<const S*>(a.W) + (size_t)r * a.V + a.v0 + w, n, x);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = 0.f;
    }
    write_pieces<PLANES>(x, a.out + (size_t)r * a.Vc + w, a.plane);
  }
}

template <class S, int PLANES>
__global__ __launch_bounds__(256) void loss_pack_w(LossPackWArgs a) {
  pack_w<S, PLANES>(a, (long long)blockIdx.x * 256 + threadIdx.x, (long long)gridDim.x * 256);
}

// What a loss lays out before its products, by workgroup:
//   lists   of a row tile's entries, sorted by the block of 32 x 32 that will hold them (a counting sort in LDS, two
//           16-bit counters a word: a block has at most 1,024 entries, as every entry of a row is of another word, and
//           a tile 32,768; the order within a block is free, each entry's result being a value of its own);
//   states  of the rows that count, in bf16 pieces, as whole row tiles with zeros behind them;
//   bias    filled up with -inf;
//   W       its first piece, where it is not read where it lies.
// Where there are few rows and entries' blocks, every workgroup finds the rows that count by itself, in LDS: a launch
// and its gap less (about 4 us) for about 2 us.
// Bound by memory where W is laid out (bf16 512 x 32,001 with 5,000 rows 21 us, 75 MB, 3.5 TB/s), else by its chain of
// dependent loads and barriers (640 rows of 1,024 9.6 us, 60 rows 6.2).
constexpr int kFindRows = 8192;
constexpr int kPackT = 1024;

template <class S, int PLANES>
__global__ __launch_bounds__(kPackT) void loss_pack(LossPackArgs a) {
  extern __shared__ uint32_t dyn[];
  __shared__ int wsum[K3_W];
  const int tid = threadIdx.x;
  int wg = blockIdx.x;
  if (wg >= a.tiles + a.states_wg) {
    wg -= a.tiles + a.states_wg;
    if (wg < a.bias_wg) {
      const int i = wg * kPackT + tid;
      if (i < a.Vp) a.bp[i] = i < a.rows.V ? a.b[i] : -INFINITY;
    } else {
      pack_w<S, PLANES>(a.w, (long long)(wg - a.bias_wg) * kPackT + tid, (long long)a.w_wg * kPackT);
    }
    return;
  }
  const int32_t* map = a.rows.map;
  int rows;
  if (a.find_rows) {
    int* own = reinterpret_cast<int*>(dyn);
    const bool tell = wg == 0;
    if (tell)
      for (int n = tid; n < a.rows.N; n += kPackT)
        if (!row_counts(a.rows, n)) a.rows.inv[n] = -1;
    rows = compact_entries_pass(
        a.rows.N, [&](int n) { return row_counts(a.rows, n); },
        [&](int c, int n) {
          own[c] = n;
          if (tell) {
            a.rows.map[c] = n;
            a.rows.inv[n] = c;
          }
        },
        wsum);
    if (tell && tid == 0) *a.rows.count = rows;
    map = own;
    __syncthreads();
  } else {
    rows = *a.rows.count;
  }
  const int R = loss_row_tiles(rows, a.BN);
  if (wg < a.tiles) {
    const int rt = wg, K = a.rows.K;
    if (rt >= R) return;
    const int here = min(a.BN, rows - rt * a.BN);
    if (a.rowp)
      for (int r = tid; r < a.BN; r += kPackT) {
        float2 v = make_float2(INFINITY, 0.f);  // no row: probabilities of zero
        if (r < here) {
          const int row = map[rt * a.BN + r];
          v = make_float2(a.lse[row], a.grad[row] * a.grad_scale);
        }
        a.rowp[rt * a.BN + r] = v;
      }
    // counter i (list i - 1) in the halves of hist[i / 2]
    uint32_t* hist = dyn + (a.find_rows ? (a.rows.N + 1) / 2 * 2 : 0);
    const int words = a.nb / 2 + 1;  // nb is even
    for (int i = tid; i < words; i += kPackT) hist[i] = 0;
    __syncthreads();
    const int wtm = loss_wtm(a.BN), wtn = loss_wtn(a.BN), NB = wtn / 32, blocks = loss_blocks(a.BN);
    // a thread's entries: j of rows r0, r0 + step, ...
    const int kp = K <= 1 ? 1 : 1 << (32 - __builtin_clz(K - 1));
    const int j = tid & (kp - 1), r0 = tid / kp, step = kPackT / kp;
    auto each = [&](auto use) {
      if (j < K)
        for (int r = r0; r < here; r += 4 * step) {
          int row[4], t[4];  // four loads under way
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            row[u] = r + u * step < here ? map[rt * a.BN + r + u * step] : -1;
            t[u] = row[u] >= 0 ? a.rows.token[(size_t)row[u] * K + j] : -1;
          }
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (t[u] >= 0 && t[u] < a.rows.V) {
              const int ru = r + u * step, second = ru >= wtn;  // of the wave's rows
              const int blk = ((t[u] & (wtm - 1)) >> 5) * NB + ((ru - (second ? wtn : 0)) >> 5);
              use(ru, row[u], t[u], ((second ? a.words0 : 0) + t[u] / wtm) * blocks + blk);
            }
        }
    };
    each([&](int, int, int, int list) { atomicAdd(&hist[(list + 1) >> 1], ((list + 1) & 1) ? 1u << 16 : 1u); });
    __syncthreads();
    // counters to first items: hist[i] becomes the sum of the counters up to i
    {
      const int per = (words + kPackT - 1) / kPackT, i0 = min(words, tid * per), i1 = min(words, i0 + per);
      int sum = 0;
      for (int i = i0; i < i1; ++i) sum += (hist[i] & 0xffffu) + (hist[i] >> 16);
      int total;
      int at = block_excl_scan(sum, wsum, &total);
      for (int i = i0; i < i1; ++i) {
        const int lo = at + (hist[i] & 0xffffu), hi = lo + (hist[i] >> 16);
        hist[i] = (uint32_t)lo | (uint32_t)hi << 16;
        at = hi;
      }
    }
    __syncthreads();
    uint32_t* offs = reinterpret_cast<uint32_t*>(a.offs + (size_t)rt * (a.nb + 2));
    for (int i = tid; i < words; i += kPackT) offs[i] = hist[i];
    __syncthreads();
    LossItem* items = a.items + (size_t)rt * a.BN * K;
    each([&](int r, int row, int t, int list) {
      const uint32_t before = atomicAdd(&hist[list >> 1], (list & 1) ? 1u << 16 : 1u);
      const int at = (list & 1) ? before >> 16 : before & 0xffffu;
      const int reg = 4 * ((t >> 3) & 3) + (t & 3), l = 32 * ((t >> 2) & 1) + (r & 31);
      const float part = a.rows.part ? a.rows.part[(size_t)row * K + j] : a.rows.target_part;
      items[at] = {reg << 8 | l, a.rowp ? __float_as_int(part) : (rt * a.BN + r) * K + j};
    });
    return;
  }
  const int chunks = a.Hp / 8, H = a.rows.H;
  const long long total = (long long)R * a.BN * chunks;
  for (long long i = (long long)(wg - a.tiles) * kPackT + tid; i < total; i += (long long)a.states_wg * kPackT) {
    const int c = (int)(i / chunks), h0 = (int)(i % chunks) * 8;
    float x[8];
    if (c < rows && h0 < H) {
      load8(static_cast<const S*>(a.h) + (size_t)map[c] * H + h0, H - h0, x);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = 0.f;
    }
    write_pieces<PLANES>(x, a.ph + (size_t)c * a.Hp + h0, a.ph_plane);
  }
}

// Bound by its chain of dependent loads (640 rows of 85 splits 5.3 us, 8,192 of 8 7.9).
// loss and log-sum-exp of every row, a wave each: M = max m, S = sum s e^((m - M) / T) over all splits, lse = M / T + ln S.
__global__ __launch_bounds__(256) void loss_finish(LossFinishArgs a) {
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.rows.N) return;
  const int c = a.rows.inv[row], K = a.rows.K;
  if (c < 0) {
    if (lane == 0) a.loss[row] = a.lse[row] = 0.f;
    return;
  }
  const int R = loss_row_tiles(*a.rows.count, a.BN);
  const int P = loss_splits(a.grid, R, a.vt_piece), last = loss_splits(a.grid, R, a.vt_last);
  float M = kStatInit, S = 0.f, X = 0.f;
  for (int p = 0; p < a.pieces; ++p) {
    const int here = p + 1 < a.pieces ? P : last;
    for (int i = lane; i < here; i += 64) {
      const size_t at = p * a.stat_piece + (size_t)c * here + i;
      const float2 v = a.stat[at];
      const float m = fmaxf(M, v.x);
      S = S * exp2f((M - m) * a.scale) + v.y * exp2f((v.x - m) * a.scale);
      M = m;
      if (a.sumx) X += a.sumx[at];
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float mo = __shfl_xor(M, d, 64), so = __shfl_xor(S, d, 64);
    X += __shfl_xor(X, d, 64);
    const float m = fmaxf(M, mo);
    S = S * exp2f((M - m) * a.scale) + so * exp2f((mo - m) * a.scale);
    M = m;
  }
  const float lse = M * a.inv_t + logf(S);
  float dot = 0.f;
  for (int j = lane; j < K; j += 64) {
    const int t = a.rows.token[(size_t)row * K + j];
    if (t < 0 || t >= a.rows.V) continue;
    const float part = a.rows.part ? a.rows.part[(size_t)row * K + j] : a.rows.target_part;
    if (part != 0.f) dot += part * a.xt[(size_t)c * K + j];  // of no weight: also where x = -inf
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) dot += __shfl_xor(dot, d, 64);
  if (lane == 0) {
    float l = lse - dot * a.inv_t - a.rest * X;
    if (a.known) l += a.known[row];
    a.loss[row] = l * a.t2;
    a.lse[row] = lse;
  }
}

__global__ __launch_bounds__(1024) void loss_db(LossBiasArgs a) {
  __shared__ float sums[1024];
  sum_bias(a, blockIdx.x, sums);
}

__global__ __launch_bounds__(256) void loss_zero(uint16_t* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}

hipError_t launch_loss_zero(void* p, size_t bytes, hipStream_t st) {
  loss_zero<<<dim3(1024), dim3(256), 0, st>>>(static_cast<uint16_t*>(p), bytes / 2);
  return hipGetLastError();
}

hipError_t launch_loss_teacher(const LossTeacherArgs& a, hipStream_t st) {
  loss_teacher<<<dim3((a.N + 3) / 4), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_loss_rows(const LossRows& a, hipStream_t st) {
  loss_rows<<<dim3(1), dim3(K3_T), 0, st>>>(a);
  return hipGetLastError();
}

bool loss_finds_rows(int N, int nb) { return N <= kFindRows && (size_t)N * 4 + (size_t)nb * 2 <= 60 * 1024; }

hipError_t launch_loss_pack(bool bf16, LossPackArgs a, hipStream_t st) {
  const long long copies = (long long)loss_row_tiles(a.rows.N, a.BN) * a.BN * (a.Hp / 8);
  a.states_wg = (int)std::min<long long>((copies + kPackT - 1) / kPackT, 512);
  a.bias_wg = (a.Vp + kPackT - 1) / kPackT;
  a.w_wg = a.w.out ? (int)std::min<long long>(((long long)a.w.Hk * (a.w.Vc / 8) + kPackT - 1) / kPackT, 2048) : 0;
  const dim3 gr(a.tiles + a.states_wg + a.bias_wg + a.w_wg), th(kPackT);
  const size_t lds = ((size_t)(a.find_rows ? (a.rows.N + 1) / 2 * 2 : 0) + a.nb / 2 + 1) * 4;
  const void* f = bf16 ? reinterpret_cast<const void*>(loss_pack<uint16_t, 1>) : reinterpret_cast<const void*>(loss_pack<float, 3>);
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  if (bf16)
    loss_pack<uint16_t, 1><<<gr, th, lds, st>>>(a);
  else
    loss_pack<float, 3><<<gr, th, lds, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_loss_pack_w(bool bf16, const LossPackWArgs& a, hipStream_t st) {
  const long long chunks = (long long)a.Hk * (a.Vc / 8);
  const dim3 gr((unsigned)((chunks + 255) / 256 < 8192 ? (chunks + 255) / 256 : 8192));
  if (bf16)
    loss_pack_w<uint16_t, 1><<<gr, dim3(256), 0, st>>>(a);
  else
    loss_pack_w<float, 3><<<gr, dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_loss_finish(const LossFinishArgs& a, hipStream_t st) {
  loss_finish<<<dim3((a.rows.N + 3) / 4), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_loss_db(const LossBiasArgs& a, hipStream_t st) {
  loss_db<<<dim3((a.V + 63) / 64), dim3(1024), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace kb
