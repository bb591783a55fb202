// Logits of the output layer's losses and what becomes of them, tile by tile: they are never stored.
//
// forward: Algorithm 4's running (max, sum of exp) of every row over the workgroup's words, the sum of the logits
// where labels are smoothed, and the logits of the rows' entries (their targets, or the teacher's words).
//
// gradient: dx = g (p - rest - part), p = exp(x / T - lse) from the log-sum-exp that the forward pass left; rounded to
// bf16 once, as the operand of the two products that follow (float32: three bf16 pieces, to 2^-24), and before that
// summed over the rows for the bias.
//
// Words are the M side: a lane has 64 (small tiles: 32) words of each of its rows, so statistics need no exchange
// until the end.  The accumulators start at the bias; words that only fill the last tile up start at -inf.
// Entries were sorted into a list for each wave's part of each tile: the wave goes through its few, reading them with
// scalar loads (about 21 for 256 x 256 at 16 entries a row and 50,000 words), and picks the register by a branch.
#pragma once

#include "loss_mm.hpp"

namespace kb {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
#define KB_CONST __attribute__((address_space(4)))

// What no kernel of the same launch writes, at wave-uniform addresses: scalar loads, whose wait leaves the DMA alone.
__device__ __forceinline__ int const_int(const int32_t* p) {
  return *(const KB_CONST int32_t*)(uintptr_t)uniform_ptr(p);
}

typedef int i32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ i32x4 const_int4(const void* p) {
  return *(const KB_CONST i32x4*)(uintptr_t)uniform_ptr(p);
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

// bf16 piece `plane` of x.
__device__ __forceinline__ float piece(float x, int plane) {
  const float p0 = (float)(__bf16)x;
  if (plane == 0) return p0;
  const float r = x - p0, p1 = (float)(__bf16)r;
  return plane == 1 ? p1 : r - p1;
}

// A tile as bf16 to rows of `out` (row n of the tile at out + n * ld, words along it), through the LDS buffer `lds`
// of one stage, 32 words of every wave at a time: 16 bytes a lane, 64 in a row, where the accumulators alone would
// give eight.  write(row, word, v): rows and words of the tile, v: 8 values.
template <class T, class Write>
__device__ __forceinline__ void store_bf16(f32x16 (&acc)[T::MB][T::NB], int plane, uint32_t lds, Write write) {
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = tid >> 6, wm = wave % T::WM, wn = wave / T::WM;
  constexpr int CH = T::WM * 4;  // 16-byte chunks of a row
  static_assert(T::BN * CH * 16 <= MmGeom<T::BM>::BYTES + MmGeom<T::BN>::BYTES, "fits in a stage");
#pragma unroll
  for (int m = 0; m < T::MB; ++m) {
    lds_barrier();
#pragma unroll
    for (int n = 0; n < T::NB; ++n) {
      in_acc(acc[m][n]);
      const int row = wn * T::WTN + n * 32 + col;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bf16x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (__bf16)piece(acc[m][n][4 * i + j], plane);
        *(KB_LDS bf16x4*)(uintptr_t)(lds + (uint32_t)(row * CH + ((wm * 4 + i) ^ (row & (CH - 1)))) * 16u + half * 8u) = v;
      }
    }
    lds_barrier();
#pragma unroll
    for (int k = 0; k < T::BN * CH / 256; ++k) {
      const int at = k * 256 + tid, row = at / CH, c = at % CH;
      const bf16x8 v = *(const KB_LDS bf16x8*)(uintptr_t)(lds + (uint32_t)(row * CH + (c ^ (row & (CH - 1)))) * 16u);
      write(row, (c >> 2) * T::WTM + m * 32 + (c & 3) * 8, v);
    }
  }
}

template <class T, int PASSES>
struct LossOcc {  // workgroups that fit on a CU
  static constexpr int STAGE = MmGeom<T::BM>::BYTES + MmGeom<T::BN>::BYTES;
  static constexpr int N = 4 * STAGE <= 76 * 1024 ? 2 : 1;
};

template <class T, int PASSES, bool GRAD>
__global__ __launch_bounds__(256, (LossOcc<T, PASSES>::N)) void loss_logits(LossLogitsArgs a) {
  constexpr int MB = T::MB, NB = T::NB, BN = T::BN;
  constexpr int PLANES = PASSES > 1 ? 3 : 1;
  __shared__ __attribute__((aligned(1024))) uint8_t ring[4 * LossOcc<T, PASSES>::STAGE];
  __shared__ __attribute__((aligned(16))) float bias[4][kLossM];
  __shared__ __attribute__((aligned(16))) float2 rowp[GRAD ? BN : 1];
  __shared__ __attribute__((aligned(16))) float red[GRAD ? 1 : BN][T::WM][3];

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
  const int rows = const_int(a.count);
  const int R = loss_row_tiles(rows, BN), P = loss_splits(a.grid, R, a.vt);
  if ((int)blockIdx.x >= R * P) return;
  int rt, sp;
  loss_cell(R, P, blockIdx.x, rt, sp);
  const int nt = (a.vt - sp + P - 1) / P;

  if constexpr (GRAD) {
    for (int r = tid; r < BN; r += 256) rowp[r] = a.rowp[rt * BN + r];
    __syncthreads();
  }
  const int32_t* offs = a.offs + (size_t)rt * (a.nb + 1) + wn * a.words0 + a.wt0 + wm;
  const LossItem* items = a.items + (size_t)rt * BN * a.K;

  auto tile = [&](int t, MmSide& A, MmSide& B) {
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
  // the wave's entries of tile t: each(block, register, lane, item)
  auto entries = [&](int t, auto each) {
    const int32_t* o = offs + (sp + t * P) * (kLossM / T::WTM);
    const int lo = const_int(o), hi = const_int(o + 1);
    for (int e = lo; e < hi; ++e) {
      const i32x4 it = const_int4(items + e);
      each(it[0] >> 16, (it[0] >> 8) & 255, it[0] & 255, it);
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
  auto epi_stats = [&](int t, f32x16 (&acc)[MB][NB]) {
    const int left = a.words - (sp + t * P) * kLossM - wm * T::WTM - 4 * half;  // words from the lane's first on
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
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
          for (int r = 0; r < 16; ++r) x0 += m * 32 + 8 * (r >> 2) + (r & 3) < left ? acc[m][n][r] : 0.f;
        st_x[n] += x0;
      }
      asm volatile("" ::"v"(st_s[n]));  // one row's 64 logits in VGPRs at a time
    }
    entries(t, [&](int blk, int r, int l, const i32x4& it) {
      float x = 0.f;
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n)
          if (blk == m * NB + n) {
            in_acc(acc[m][n]);
#pragma unroll
            for (int i = 0; i < 16; ++i) x = r == i ? acc[m][n][i] : x;
          }
      if (lane == l) a.xt[it[1]] = x;
    });
  };
  auto epi_grad = [&](int t, f32x16 (&acc)[MB][NB], uint32_t lds) {
    const int v0 = (sp + t * P) * kLossM;
    const int left = a.words - v0 - wm * T::WTM - 4 * half;
    const bool ragged = v0 + kLossM > a.words && a.rest != 0.f;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const float2 rp = rowp[wn * T::WTN + n * 32 + col];  // (lse, g)
      const float off = PASSES > 1 ? rp.x : rp.x * kL2E;
      const float gr = rp.y * a.rest;
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        in_acc(acc[m][n]);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          // float32: the difference first, so that its rounding and not that of lse * log2(e) is what p sees
          const float e = PASSES > 1 ? fmaf(acc[m][n][r], a.scale, -off) * kL2E : fmaf(acc[m][n][r], a.scale, -off);
          float v = fmaf(rp.y, exp2_fast(e), -gr);
          if (ragged && m * 32 + 8 * (r >> 2) + (r & 3) >= left) v = 0.f;
          acc[m][n][r] = v;
        }
        in_acc(acc[m][n]);
      }
    }
    entries(t, [&](int blk, int r, int l, const i32x4& it) {
      const float q = __int_as_float(it[2]);
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n)
          if (blk == m * NB + n) {
            in_acc(acc[m][n]);
            const float d = lane == l ? q * rowp[wn * T::WTN + n * 32 + col].y : 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][n][i] -= r == i ? d : 0.f;
            in_acc(acc[m][n]);
          }
    });
    if (a.dbp) {
      // over the wave's rows: its blocks in registers, then the 32 lanes by halving the words a lane keeps
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        float s[16];
#pragma unroll
        for (int n = 0; n < NB; ++n) in_acc(acc[m][n]);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = acc[m][0][r];
#pragma unroll
          for (int n = 1; n < NB; ++n) s[r] += acc[m][n][r];
        }
#pragma unroll
        for (int w = 8; w >= 1; w >>= 1) {
          const bool up = (col & (2 * w)) != 0;
#pragma unroll
          for (int r = 0; r < w; ++r) {
            const float keep = up ? s[r + w] : s[r], give = up ? s[r] : s[r + w];
            s[r] = keep + __shfl_xor(give, 2 * w, 64);
          }
        }
        s[0] += __shfl_xor(s[0], 1, 64);
        const int r = col >> 1;  // bits 4..1 of the lane chose the word's bits 3..0
        if ((col & 1) == 0)
          a.dbp[(size_t)(rt * T::WN + wn) * a.db_ld + a.db0 + v0 + wm * T::WTM + m * 32 + 8 * (r >> 2) + 4 * half + (r & 3)] =
              s[0];
      }
    }
#pragma unroll 1
    for (int pl = 0; pl < PLANES; ++pl) {
      uint16_t* out = a.g + pl * a.g_plane + (size_t)rt * BN * a.gld + v0;
      store_bf16<T>(acc, pl, lds, [&](int row, int word, const bf16x8& v) {
        *reinterpret_cast<bf16x8*>(out + (size_t)row * a.gld + word) = v;
      });
    }
  };
  auto epi = [&](int t, f32x16 (&acc)[MB][NB], uint32_t lds) {
    if constexpr (GRAD)
      epi_grad(t, acc, lds);
    else
      epi_stats(t, acc);
  };
  mm_run<T, true, false, PASSES == 1, PASSES>(lds_addr(ring), nt, a.Hk / kLossStage, tile, init, epi);

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

template <int PASSES>
hipError_t launch_loss_logits_t(bool grad, int BN, const LossLogitsArgs& a, int blocks, hipStream_t st) {
  const dim3 gr(blocks), th(256);
  if (grad) {
    switch (BN) {
      case 256: loss_logits<LossT256, PASSES, true><<<gr, th, 0, st>>>(a); break;
      case 128: loss_logits<LossT128, PASSES, true><<<gr, th, 0, st>>>(a); break;
      case 64: loss_logits<LossT64, PASSES, true><<<gr, th, 0, st>>>(a); break;
      default: loss_logits<LossT32, PASSES, true><<<gr, th, 0, st>>>(a); break;
    }
  } else {
    switch (BN) {
      case 256: loss_logits<LossT256, PASSES, false><<<gr, th, 0, st>>>(a); break;
      case 128: loss_logits<LossT128, PASSES, false><<<gr, th, 0, st>>>(a); break;
      case 64: loss_logits<LossT64, PASSES, false><<<gr, th, 0, st>>>(a); break;
      default: loss_logits<LossT32, PASSES, false><<<gr, th, 0, st>>>(a); break;
    }
  }
  return hipGetLastError();
}

}  // namespace kb
