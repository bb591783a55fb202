// Logits of the output layer's losses and what becomes of them, tile by tile: they are never stored.
//
// forward: Algorithm 4's running (max, sum of exp) of every row over the workgroup's words, the sum of the logits
// where labels are smoothed, and the logits of the rows' entries (their targets, or the teacher's words).
//
// gradient: dx = g (p - rest - part), p = exp(x / T - lse) from the log-sum-exp that the forward pass left; summed over the
// rows in float32 for the bias, and then rounded to bf16 as the operand of the two products that follow, a rounding as
// large as the one of their bf16 results.  Of at most 128 rows, whose gradients a few dlogits dominate (and whose
// time the reading of W and the writing of dW do), it is kept in two bf16 pieces, to 2^-17; of float32 operands in
// three, to 2^-24.
//
// Words are the M side: a lane has 64 (small tiles: 32) words of each of its rows, so statistics need no exchange
// until the end.  The accumulators start at the bias; words that only fill the last tile up start at -inf.
// Entries were sorted into lists by the 32 x 32 block that holds their logits.  A block with entries goes through LDS of
// the wave's own, from its accumulators to the entries' lanes or the other way: picking registers for one entry after
// the other took 1.5 ms more for 4,096 rows of 64 words of 60,000, as a teacher's words cluster where the vocabulary's
// frequent words are (half of the 64 in one tile of 256).
//
// Bound by the main loop (loss_mm.hpp) and, of 512 states and fewer, by the epilogue beside it: an exponential, three
// other operations and an accumulator's read for each logit, 3 of a tile's 18 us there.  8,192 x 1,024 x 90,000: the
// forward pass 1,293 us (1.17 PFLOP/s, matrix cores 58% busy), the gradient's 1,628 in eleven pieces (0.93, and 1.5 GB of
// dlogits written); 640 x 512 x 30,000 of float32 140 and 168.
#pragma once

#include "loss_load.hpp"
#include "loss_mm.hpp"

namespace kb {

typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
#define KB_CONST __attribute__((address_space(4)))

// What no kernel of the same launch writes, at wave-uniform addresses: scalar loads, whose wait leaves the DMA alone.
__device__ __forceinline__ int const_int(const int32_t* p) {
  return *(const KB_CONST int32_t*)(uintptr_t)uniform_ptr(p);
}

// Workgroup b of the R x P cells: those of an XCD (every eighth workgroup) are neighbours, groups of four row tiles
// walked split by split, so that one L2 sees the tiles of W asked for by several row tiles at about the same time.
__device__ __forceinline__ void loss_cell(int R, int P, int b, int& rt, int& sp) {
  const int T = R * P, x = b & 7, j = b >> 3;
  const int c = x * (T >> 3) + min(x, T & 7) + j;
  constexpr int GR = 4;
  const int full = R / GR, gcells = GR * P;
  int rg = c / gcells, gr = GR, q = c - rg * gcells;
  if (rg >= full) {
    gr = R - full * GR;
    rg = full;
    q = c - full * gcells;
  }
  sp = q / gr;
  rt = rg * GR + (q - sp * gr);
}

// 32 words of a wave's rows as bf16, through LDS of the wave's own (64 bytes a row, in 16-byte chunks that are swizzled
// by the row), to rows of memory: 16 bytes a lane, 64 in one piece, where the accumulators alone would give eight.
// Waves need not wait for each other: a wave's LDS operations are done in their order.
// value(n, r): register r of the rows of block n; write(row, word, v): within the wave's part, v: 8 values.
template <class T, class Value, class Write>
__device__ __forceinline__ void store_rows(uint32_t mine, Value value, Write write) {
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
#pragma unroll
  for (int n = 0; n < T::NB; ++n) {
    const int row = n * 32 + col;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = value(n, 4 * i + j);
      *(KB_LDS bf16x4*)(uintptr_t)(mine + (uint32_t)(row * 64 + (i ^ hswz(row)) * 16 + half * 8)) = v;
    }
  }
#pragma unroll
  for (int k = 0; k < T::WTN / 16; ++k) {
    const int row = k * 16 + (lane >> 2), c = lane & 3;
    const bf16x8 v = *(const KB_LDS bf16x8*)(uintptr_t)(mine + (uint32_t)(row * 64 + (c ^ hswz(row)) * 16));
    write(row, c * 8, v);
  }
}

// s[0 .. 16) summed over each half's 32 lanes: lane i gets value (i & 31) / 2.  Rows of 16 lanes swap halves of the
// values; within a row, lanes keep half of what is left and take their mirror image's other half.
__device__ __forceinline__ float sum32(float (&s)[16], int lane) {
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(s[r]), __float_as_uint(s[r + 8]), false, false);
    s[r] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  const bool b3 = (lane & 8) != 0, b2 = (lane & 4) != 0, b1 = (lane & 2) != 0;
#pragma unroll
  for (int r = 0; r < 4; ++r) s[r] = (b3 ? s[r + 4] : s[r]) + dpp_of<0x140>(b3 ? s[r] : s[r + 4]);  // row_mirror
#pragma unroll
  for (int r = 0; r < 2; ++r) s[r] = (b2 ? s[r + 2] : s[r]) + dpp_of<0x141>(b2 ? s[r] : s[r + 2]);  // row_half_mirror
  s[0] = (b1 ? s[1] : s[0]) + dpp_of<0x1b>(b1 ? s[0] : s[1]);                                       // quad_perm 3 2 1 0
  return s[0] + dpp_of<0xb1>(s[0]);                                                                 // quad_perm 1 0 3 2
}

// As many entries of a wave's part of a tile are read by scalar loads.
constexpr int kFewEntries = 4;

template <class T>
struct LossOcc {  // workgroups that fit on a CU
  static constexpr int STAGE = MmGeom<T::BM>::BYTES + MmGeom<T::BN>::BYTES;
  static constexpr int N = 4 * STAGE <= 76 * 1024 ? 2 : 1;
};

// PASSES: 1 (bf16 operands) or 6 (float32); PLANES: bf16 pieces of the dlogits, 0 for the forward pass.
template <class T, int PASSES, int PLANES>
__global__ __launch_bounds__(256, (LossOcc<T>::N)) void loss_logits(LossLogitsArgs a) {
  constexpr int MB = T::MB, NB = T::NB, BN = T::BN;
  constexpr bool GRAD = PLANES > 0;
  constexpr int NBLK = MB * NB;
  __shared__ __attribute__((aligned(1024))) uint8_t ring[4 * LossOcc<T>::STAGE];
  __shared__ __attribute__((aligned(16))) float bias[4][kLossM];
  __shared__ __attribute__((aligned(16))) float2 rowp[GRAD ? BN : 1];
  __shared__ __attribute__((aligned(16))) float red[GRAD ? 1 : BN][T::WM][3];
  // the gradient's entries have LDS of their own, but for the tile of which two workgroups then fit no more
  constexpr bool APART = GRAD && LossOcc<T>::N == 1;
  __shared__ __attribute__((aligned(16))) uint8_t apart[APART ? 4 * 32 * 36 * 4 : 16];

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
  const int rows = const_int(a.count);
  const int R = loss_row_tiles(rows, BN), P = loss_splits(a.grid, R, a.vt);
  if ((int)blockIdx.x >= R * P) return;
  int rt, sp;
  loss_cell(R, P, blockIdx.x, rt, sp);
  const int nt = (a.vt - sp + P - 1) / P;
  using Args = LossLogitsArgs;

  if constexpr (GRAD) {
    for (int r = tid; r < BN; r += 256) rowp[r] = a.rowp[rt * BN + r];
    __syncthreads();
  }

  auto tile = [&](int t, MmSide& A, MmSide& B) {
    const auto& a = *args_again<Args>();
    const int v0 = (sp + t * P) * kLossM;
    A = {a.A + v0, a.lda, a.a_plane, a.a_cols - v0, 0};
    B = {a.ph + (size_t)rt * BN * a.Hp, a.Hp, a.ph_plane, 0, 0};
    if (wave == 0) dma16(a.b + v0 + lane * 4, lds_addr(&bias[t & 3][0]));
  };
  auto init = [&](int t, f32x16 (&acc)[MB][NB]) {
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      f32x16 bv;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 b = *reinterpret_cast<const float4*>(&bias[t & 3][wm * T::WTM + m * 32 + 8 * i + 4 * half]);
        bv[4 * i + 0] = b.x;
        bv[4 * i + 1] = b.y;
        bv[4 * i + 2] = b.z;
        bv[4 * i + 3] = b.w;
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        acc[m][n] = bv;
        in_acc(acc[m][n]);
      }
    }
  };
  // The wave's entries of a tile, block by block (m, n).  The first 256 are held four a lane, loaded as the epilogue
  // begins (a few: by scalar loads, which do not wait for the DMA); those of a block move between the accumulators and
  // their lanes through LDS of the wave's own, the block's 32 rows 36 floats apart.
  struct Entries {
    const LossItem* items;
    uint32_t offs[NBLK / 2 + 1];  // two a word: first entries of the blocks, the end of the last one
    int lo, n;
    int payload[4];
    uint32_t at[4];
  };
  auto entry_at = [&](uint32_t mine, int code) {
    const int r = code >> 8, l = code & 255;
    return mine + (uint32_t)((l & 31) * 36 + 8 * (r >> 2) + 4 * (l >> 5) + (r & 3)) * 4u;
  };
  auto load_entries = [&](int t, uint32_t mine, Entries& e) {
    const auto& a = *args_again<Args>();
    const int list = wn * a.words0 + a.wt0 + wm + (sp + t * P) * (kLossM / T::WTM);
    const uint16_t* o = a.offs + (size_t)rt * (a.nb + 2) + (size_t)list * NBLK;
    e.items = a.items + (size_t)rt * BN * a.K;
#pragma unroll
    for (int i = 0; i <= NBLK / 2; ++i) e.offs[i] = (uint32_t)const_int(reinterpret_cast<const int32_t*>(o) + i);
    e.lo = e.offs[0] & 0xffffu;
    e.n = (int)(e.offs[NBLK / 2] & 0xffffu) - e.lo;
    if (e.n <= 0) return;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      e.payload[u] = 0;
      e.at[u] = mine;
    }
    if (e.n <= kFewEntries) {
      for (int i = 0; i < e.n; ++i) {
        const int code = const_int(&e.items[e.lo + i].code), payload = const_int(&e.items[e.lo + i].payload);
        if (lane == i) {
          e.at[0] = entry_at(mine, code);
          e.payload[0] = payload;
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (u * 64 + lane < e.n) {
          const LossItem it = e.items[e.lo + u * 64 + lane];
          e.at[u] = entry_at(mine, it.code);
          e.payload[u] = it.payload;
        }
    }
  };
  auto block_has = [&](const Entries& e, int b, int& lo, int& hi) {  // first and end within the list
    lo = (int)((b & 1 ? e.offs[b / 2] >> 16 : e.offs[b / 2] & 0xffffu)) - e.lo;
    hi = (int)(((b + 1) & 1 ? e.offs[(b + 1) / 2] >> 16 : e.offs[(b + 1) / 2] & 0xffffu)) - e.lo;
    return hi > lo;
  };
  auto each_entry = [&](const Entries& e, uint32_t mine, int lo, int hi, auto use) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (u * 64 + lane >= lo && u * 64 + lane < hi) use(e.at[u], e.payload[u]);
    for (int i = max(lo, 256) + lane; i < hi; i += 64) {
      const LossItem it = e.items[e.lo + i];
      use(entry_at(mine, it.code), it.payload);
    }
  };

  float st_m[NB], st_s[NB], st_x[NB];
  if constexpr (!GRAD) {
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      st_m[n] = kStatInit;
      st_s[n] = st_x[n] = 0.f;
    }
  }
  auto epi_stats = [&](int t, f32x16 (&acc)[MB][NB], uint32_t lds) {
    const auto& a = *args_again<Args>();
    const int left = a.words - (sp + t * P) * kLossM - wm * T::WTM - 4 * half;  // words from the lane's first on
    const bool ragged = (sp + t * P + 1) * kLossM > a.words;
    const uint32_t mine = lds + wave * (32 * 36 * 4), words = mine + (uint32_t)(col * 36 + 4 * half) * 4u;
    Entries e;
    load_entries(t, mine, e);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int m = 0; m < MB; ++m) in_acc(acc[m][n]);
      float m0 = acc[0][n][0], m1 = acc[0][n][1];
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          m0 = fmaxf(m0, acc[m][n][r]);
          m1 = fmaxf(m1, acc[m][n][r + 1]);
        }
      const float mnew = fmaxf(st_m[n], fmaxf(m0, m1));
      const float ml2 = mnew * a.scale;
      float s0 = st_s[n] * exp2_fast((st_m[n] - mnew) * a.scale), s1 = 0.f;
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          s0 += exp2_fast(fmaf(acc[m][n][r], a.scale, -ml2));
          s1 += exp2_fast(fmaf(acc[m][n][r + 1], a.scale, -ml2));
        }
      st_s[n] = s0 + s1;
      st_m[n] = mnew;
      if (a.sumx) {
        float x0 = 0.f;
        if (ragged) {
          int l = left;
          asm volatile("" : "+v"(l));  // the comparisons of every row anew, not kept in 128 scalar registers
#pragma unroll
          for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) x0 += m * 32 + 8 * (r >> 2) + (r & 3) < l ? acc[m][n][r] : 0.f;
        } else {
#pragma unroll
          for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) x0 += acc[m][n][r];
        }
        st_x[n] += x0;
      }
      if (e.n > 0) {
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          int lo, hi;
          if (!block_has(e, m * NB + n, lo, hi)) continue;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *(KB_LDS f32x4v*)(uintptr_t)(words + i * 32u) =
                f32x4v{acc[m][n][4 * i], acc[m][n][4 * i + 1], acc[m][n][4 * i + 2], acc[m][n][4 * i + 3]};
          each_entry(e, mine, lo, hi, [&](uint32_t at, int slot) { a.xt[slot] = *(const KB_LDS float*)(uintptr_t)at; });
        }
      }
      asm volatile("" ::"v"(st_s[n]));  // one row's 64 logits in VGPRs at a time
    }
  };
  // dlogits, 32 words at a time: from the accumulators through the entries, the bias' sums and the rounding to memory
  auto epi_grad = [&](int t, f32x16 (&acc)[MB][NB], uint32_t lds) {
    const auto& a = *args_again<Args>();
    const int v0 = (sp + t * P) * kLossM;
    const int left = a.words - v0 - wm * T::WTM - 4 * half;
    const bool ragged = v0 + kLossM > a.words && a.rest != 0.f;
    static_assert(4 * T::WTN * 64 <= LossOcc<T>::STAGE && 4 * 32 * 36 * 4 <= LossOcc<T>::STAGE, "fit in a stage");
    const uint32_t mine = (APART ? lds_addr(apart) : lds) + wave * (32 * 36 * 4);
    const uint32_t words = mine + (uint32_t)(col * 36 + 4 * half) * 4u;
    Entries e;
    load_entries(t, mine, e);
    float off[NB], g[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const float2 rp = rowp[wn * T::WTN + n * 32 + col];  // (lse, g)
      off[n] = PASSES > 1 ? rp.x : rp.x * kL2E;
      g[n] = rp.y;
    }
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      float x[NB][16];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        in_acc(acc[m][n]);
        const float gr = g[n] * a.rest;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          // float32: the difference first, so that its rounding and not that of lse * log2(e) is what p sees
          const float y = PASSES > 1 ? fmaf(acc[m][n][r], a.scale, -off[n]) * kL2E : fmaf(acc[m][n][r], a.scale, -off[n]);
          x[n][r] = fmaf(g[n], exp2_fast(y), -gr);
        }
        if (ragged) {
          int l = left;
          asm volatile("" : "+v"(l));
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (m * 32 + 8 * (r >> 2) + (r & 3) >= l) x[n][r] = 0.f;
        }
        int lo, hi;
        if (e.n > 0 && block_has(e, m * NB + n, lo, hi)) {
#pragma unroll
          for (int i = 0; i < 4; ++i) *(KB_LDS f32x4v*)(uintptr_t)(words + i * 32u) = f32x4v{0.f, 0.f, 0.f, 0.f};
          each_entry(e, mine, lo, hi, [&](uint32_t at, int q) { *(KB_LDS float*)(uintptr_t)at = __int_as_float(q); });
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4v q = *(const KB_LDS f32x4v*)(uintptr_t)(words + i * 32u);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[n][4 * i + j] = fmaf(-g[n], q[j], x[n][4 * i + j]);
          }
        }
      }
      if (a.dbp) {
        // over the wave's rows: its blocks in registers, then the 32 lanes by halving the words that a lane keeps
        float s[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = x[0][r];
#pragma unroll
          for (int n = 1; n < NB; ++n) s[r] += x[n][r];
        }
        const float sum = sum32(s, lane);
        const int r = col >> 1;  // the word whose sum the lane has: bits 4 .. 1 of the lane
        if ((lane & 1) == 0)
          a.dbp[(size_t)(rt * T::WN + wn) * a.db_ld + a.db0 + v0 + wm * T::WTM + m * 32 + 8 * (r >> 2) + 4 * half + (r & 3)] =
              sum;
      }
#pragma unroll
      for (int pl = 0; pl < PLANES; ++pl) {
        uint16_t* out = a.g + pl * a.g_plane + (size_t)(rt * BN + wn * T::WTN) * a.gld + v0 + wm * T::WTM + m * 32;
        store_rows<T>(APART ? lds + wave * (T::WTN * 64) : mine, [&](int n, int r) {
          const __bf16 v = (__bf16)x[n][r];
          if (pl + 1 < PLANES) x[n][r] -= (float)v;
          return v;
        }, [&](int row, int word, const bf16x8& v) {
          *reinterpret_cast<bf16x8*>(out + (size_t)row * a.gld + word) = v;
        });
      }
    }
  };
  constexpr int STORES = MB * PLANES * (T::WTN / 16);
  auto epi = [&](int t, f32x16 (&acc)[MB][NB], uint32_t lds) {
    if constexpr (GRAD)
      epi_grad(t, acc, lds);
    else
      epi_stats(t, acc, lds);
  };
  using Passes = std::conditional_t<PASSES == 1, MmOne, MmSix>;
  mm_run<T, true, false, PASSES == 1, Passes, STORES>(lds_addr(ring), nt, a.Hk / kLossStage, tile, init, epi);

  if constexpr (!GRAD) {
    // the row's holders: two lane halves, and the waves along the words
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const float mo = __shfl_xor(st_m[n], 32, 64), so = __shfl_xor(st_s[n], 32, 64), xo = __shfl_xor(st_x[n], 32, 64);
      const float M = fmaxf(st_m[n], mo);
      const float S = st_s[n] * exp2_fast((st_m[n] - M) * a.scale) + so * exp2_fast((mo - M) * a.scale);
      if (half == 0) {
        float* q = red[wn * T::WTN + n * 32 + col][wm];
        q[0] = M;
        q[1] = S;
        q[2] = st_x[n] + xo;
      }
    }
    __syncthreads();
    for (int r = tid; r < BN; r += 256) {
      const int row = rt * BN + r;
      if (row >= rows) continue;
      float M = red[r][0][0];
#pragma unroll
      for (int w = 1; w < T::WM; ++w) M = fmaxf(M, red[r][w][0]);
      float S = 0.f, X = 0.f;
#pragma unroll
      for (int w = 0; w < T::WM; ++w) {
        S += red[r][w][1] * exp2_fast((red[r][w][0] - M) * a.scale);
        X += red[r][w][2];
      }
      const size_t at = (size_t)row * P + sp;
      a.stat[at] = make_float2(M, S);
      if (a.sumx) a.sumx[at] = X;
    }
  }
}

// planes: of the dlogits (1 or 2 for bf16 operands, 3 for float32); 0: forward.
template <int PASSES, int PLANES>
hipError_t launch_loss_logits_p(int BN, const LossLogitsArgs& a, int blocks, hipStream_t st) {
  const dim3 gr(blocks), th(256);
  switch (BN) {
    case 256:
      if constexpr (PLANES != 2) {  // at most 128 rows have two
        loss_logits<LossT256, PASSES, PLANES><<<gr, th, 0, st>>>(a);
        break;
      }
      return hipErrorInvalidValue;
    case 192:
      if constexpr (PLANES != 2) {
        loss_logits<LossT192, PASSES, PLANES><<<gr, th, 0, st>>>(a);
        break;
      }
      return hipErrorInvalidValue;
    case 128: loss_logits<LossT128, PASSES, PLANES><<<gr, th, 0, st>>>(a); break;
    case 64: loss_logits<LossT64, PASSES, PLANES><<<gr, th, 0, st>>>(a); break;
    default: loss_logits<LossT32, PASSES, PLANES><<<gr, th, 0, st>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace kb
