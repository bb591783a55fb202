// The gradients of the output layer's losses from a piece's dlogits: dh = dx W^T over the words, dW = h^T dx over the
// rows, both with the 256-wide M side on what lies along the result's rows (states of dh, words of dW).
//
// A long axis is split where the tiles alone would not fill the card; the parts stay in the order of the registers, 16
// bytes a lane, and a join adds them up in order.  dh takes the words piece by piece and adds to its parts.
//
// Bound by the main loop: 8,192 x 1,024 x 90,000 2,553 us for both in eleven pieces (1.18 PFLOP/s, matrix cores 58% busy),
// 48 for the join.  60 x 1,024 x 50,000: by memory, dW 35 us (102 MB written), dh 26 (as much read).
#pragma once

#include "loss_bias.hpp"
#include "loss_logits.hpp"

namespace kb {

template <class T>
__device__ __forceinline__ void part_of(float* part, size_t tile, int i, f32x16& x, bool load) {
  float4* p = reinterpret_cast<float4*>(part) + (tile * (T::MB * T::NB) + i) * 4 * 256 + threadIdx.x;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (load) {
      const float4 v = p[q * 256];
      x[4 * q] = v.x, x[4 * q + 1] = v.y, x[4 * q + 2] = v.z, x[4 * q + 3] = v.w;
    } else {
      p[q * 256] = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
    }
  }
}

// One tile of a split; b: the workgroup among `cells`, dealt so that an XCD has neighbours.
__device__ __forceinline__ int xcd_cell(int cells, int b) {
  const int x = b & 7, j = b >> 3;
  return x * (cells >> 3) + min(x, cells & 7) + j;
}

// Tile c of the `cells` of dh; PASSES: 1 (bf16 operands) or 6 (float32).  Dlogits in two bf16 pieces are rows of
// their own, behind all of the first pieces', and the join adds the two rows' results.
template <class T, int PASSES>
__device__ __forceinline__ void dh_tile(const LossGradArgs& a, uint32_t ring, int R, int c) {
  const int split = c / (R * a.mt), at = c - split * (R * a.mt), rt = at / a.mt, mt = at - rt * a.mt;
  // stages of 32 words, the splits' shares of them alike
  const int stages = a.vt * (kLossM / kLossStage);
  const int s0 = (int)((long long)stages * split / a.splits), s1 = (int)((long long)stages * (split + 1) / a.splits);
  const int k0 = s0 * kLossStage, m0 = mt * kLossM;
  auto tile = [&](int, MmSide& A, MmSide& B) {
    A = {a.W + (size_t)m0 * a.ldw + k0, a.ldw, a.w_plane, a.w_rows - m0, a.words - k0};
    B = {a.g + (size_t)rt * T::BN * a.gld + k0, a.gld, a.g_plane, 0, 0};
  };
  const size_t part = (size_t)split * ((a.two > 0 ? 1 : loss_row_tiles(a.N, T::BN)) * a.mt) + at;
  auto init = [&](int, f32x16 (&acc)[T::MB][T::NB]) {
#pragma unroll
    for (int i = 0; i < T::MB * T::NB; ++i) {
      f32x16& x = acc[i / T::NB][i % T::NB];
      if (a.add) {
        part_of<T>(a.part, part, i, x, true);
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = 0.f;
      }
      in_acc(x);
    }
  };
  auto epi = [&](int, f32x16 (&acc)[T::MB][T::NB], uint32_t) {
#pragma unroll
    for (int i = 0; i < T::MB * T::NB; ++i) {
      in_acc(acc[i / T::NB][i % T::NB]);
      part_of<T>(a.part, part, i, acc[i / T::NB][i % T::NB], false);
    }
  };
  mm_run<T, false, false, true, std::conditional_t<PASSES == 1, MmOne, MmSix>, 0>(ring, 1, s1 - s0, tile, init, epi);
}

// A wave's part of a tile to rows of memory, `out` its first element, `left_rows` x `left` of which exist: 32 rows at a
// time through LDS of the wave's own, 128 or 256 bytes a row in 16-byte chunks that are swizzled by the row, and from
// there 16 bytes a lane at any element's address (written from the accumulators, 8 or 16 bytes a lane, rows of an odd
// length by single values: 1,111 x 500 x 32,001 251 us and 214; 4,096 x 1,024 x 50,000 in pieces of 64 bytes 1,475 us
// and 1,460).
template <class T, class D>
__device__ __forceinline__ void store_tile(uint32_t mine, f32x16 (&acc)[T::MB][T::NB], D* out, size_t ld, int left_rows,
                                           int left) {
  typedef D Quad __attribute__((ext_vector_type(4)));
  typedef D Chunk __attribute__((ext_vector_type(16 / sizeof(D))));
  typedef Chunk AnyChunk __attribute__((aligned(sizeof(D))));
  constexpr int WORDS = 16 / sizeof(D);                 // of a chunk
  constexpr int CH = T::BN == 256 ? 16 : 8;             // chunks of a row
  constexpr int BLK = 32 / WORDS, MG = CH / BLK;        // chunks of a block, blocks of a row
  static_assert(4 * 32 * CH * 16 <= LossOcc<T>::STAGE && T::MB % MG == 0, "fits in a stage");
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31, c = lane % CH;
  auto at = [&](int row, int chunk) { return mine + (uint32_t)(row * CH * 16 + (chunk ^ (row & (CH - 1))) * 16); };
#pragma unroll
  for (int m = 0; m < T::MB; m += MG) {
    const int word = m * 32 + c * WORDS;
#pragma unroll
    for (int n = 0; n < T::NB; ++n) {
#pragma unroll
      for (int u = 0; u < MG; ++u) {
        const f32x16& x = acc[m + u][n];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          Quad v;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = (D)x[4 * i + j];
          const int byte = (8 * i + 4 * half) * sizeof(D);  // within the block's row
          *(KB_LDS Quad*)(uintptr_t)(at(col, u * BLK + byte / 16) + byte % 16) = v;
        }
      }
#pragma unroll
      for (int k = 0; k < CH / 2; ++k) {
        const int r = k * (64 / CH) + lane / CH, row = n * 32 + r;
        const Chunk v = *(const KB_LDS Chunk*)(uintptr_t)at(r, c);
        D* to = out + (size_t)row * ld + word;
        if (row >= left_rows) continue;
        if (left - word >= WORDS) {
          *reinterpret_cast<AnyChunk*>(to) = v;
        } else {
#pragma unroll
          for (int q = 0; q < WORDS; ++q)
            if (q < left - word) to[q] = v[q];
        }
      }
    }
  }
}

// Tiles c, c + step, ... below `cells` of the tiles and splits of dW (all the splits of a workgroup's tiles have the
// same stages: it takes several only where there is one split); PASSES: 1 (bf16 operands), 2 (the dlogits in two bf16
// pieces) or 6 (float32).
template <class T, int PASSES>
__device__ __forceinline__ void dw_tile(const LossGradArgs& a, uint32_t ring, int rows, int first, int step, int cells) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
  const int stages = (rows + kLossStage - 1) / kLossStage;
  const int tiles = a.mt * a.ntn, nt = (cells - first + step - 1) / step;
  // (a division leaves its quotient in a vector register)
  auto stage0 = [&](int split) { return __builtin_amdgcn_readfirstlane((int)((long long)stages * split / a.splits)); };
  auto stages_of = [&](int c) { return stage0(c / tiles + 1) - stage0(c / tiles); };
  // the state tiles of the same words next to each other: they read the same dlogits
  auto place = [&](int t, int& m0, int& n0) {
    const int at = __builtin_amdgcn_readfirstlane((first + t * step) % tiles);
    const int mt = __builtin_amdgcn_readfirstlane(at / a.ntn);
    m0 = mt * kLossM;
    n0 = (at - mt * a.ntn) * T::BN;
  };
  auto tile = [&](int t, MmSide& A, MmSide& B) {
    int m0, n0;
    place(t, m0, n0);
    const size_t k0 = (size_t)stage0((first + t * step) / tiles) * kLossStage;
    A = {a.g + k0 * a.gld + m0, a.gld, a.g_plane, 0, 0};
    B = {a.ph + k0 * a.Hp + n0, a.Hp, a.ph_plane, 0, 0};
  };
  auto init = [&](int, f32x16 (&acc)[T::MB][T::NB]) {
#pragma unroll
    for (int i = 0; i < T::MB * T::NB; ++i) {
      f32x16& x = acc[i / T::NB][i % T::NB];
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = 0.f;
      in_acc(x);
    }
  };
  auto epi = [&](int t, f32x16 (&acc)[T::MB][T::NB], uint32_t lds) {
    int m0, n0;
    place(t, m0, n0);
    if (a.part) {
#pragma unroll
      for (int i = 0; i < T::MB * T::NB; ++i) {
        in_acc(acc[i / T::NB][i % T::NB]);
        part_of<T>(a.part, first + t * step, i, acc[i / T::NB][i % T::NB], false);
      }
      return;
    }
    using D = std::conditional_t<PASSES <= 2, __bf16, float>;
#pragma unroll
    for (int i = 0; i < T::MB * T::NB; ++i) in_acc(acc[i / T::NB][i % T::NB]);
    const int r0 = n0 + wn * T::WTN, w0 = m0 + wm * T::WTM;
    store_tile<T>(lds + wave * (LossOcc<T>::STAGE / 4 / 16 * 16), acc, static_cast<D*>(a.out) + (size_t)r0 * a.V + w0, a.V,
                  a.H - r0, a.words - w0);
  };
  mm_run<T, true, true, false, std::conditional_t<PASSES == 1, MmOne, std::conditional_t<PASSES == 2, MmTwoA, MmSix>>, 0>(
      ring, nt, stages_of(first), tile, init, epi);
}

template <class T, int PASSES>
__global__ __launch_bounds__(256, (LossOcc<T>::N)) void loss_dh(LossGradArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t ring[4 * LossOcc<T>::STAGE];
  const int R = a.two > 0 ? 1 : loss_row_tiles(const_int(a.count), T::BN), cells = a.splits * R * a.mt;
  if ((int)blockIdx.x < cells) dh_tile<T, PASSES>(a, lds_addr(ring), R, xcd_cell(cells, blockIdx.x));
}

template <class T, int PASSES>
__global__ __launch_bounds__(256, (LossOcc<T>::N)) void loss_dw(LossGradArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t ring[4 * LossOcc<T>::STAGE];
  dw_tile<T, PASSES>(a, lds_addr(ring), const_int(a.count), xcd_cell(gridDim.x, blockIdx.x), gridDim.x,
                     a.splits * a.mt * a.ntn);
}

// Both in one launch, the longer tiles of dh (TH) first: neither has to fill the card by itself.
template <class TH, class T, int PASSES>
__global__ __launch_bounds__(256, (LossOcc<T>::N)) void loss_both(LossGradArgs h, LossGradArgs w) {
  __shared__ __attribute__((aligned(1024))) uint8_t ring[4 * LossOcc<T>::STAGE];
  const int rows = const_int(h.count), R = loss_row_tiles(rows, TH::BN);
  const int ch = h.splits * R * h.mt, cw = w.splits * w.mt * w.ntn;
  if ((int)blockIdx.x < ch)
    dh_tile<TH, PASSES>(h, lds_addr(ring), R, xcd_cell(ch, blockIdx.x));
  else if ((int)blockIdx.x < ch + cw)
    dw_tile<T, PASSES>(w, lds_addr(ring), rows, xcd_cell(cw, blockIdx.x - ch), cw, cw);
}

// Workgroups of a join, of at most 2^22 tiles (2^22 rows of 2^16 states) and 64 a tile.
template <class T>
__host__ __device__ constexpr int loss_join_blocks(int tiles) {
  return tiles * (T::MB * T::NB * 4);
}

// The parts of a result added up in order and rounded once.  A workgroup takes a quarter of the registers of one block of
// 32 x 32 of every wave of a tile: four groups of 256 threads add up every fourth part each, then the four sums.
// Behind them, workgroups that fill the rows of dh that do not count with zeros, and some that add up the bias' sums.
template <class T, class D>
__global__ __launch_bounds__(1024) void loss_join(LossJoinArgs a, LossJoinMore more) {
  __shared__ float4 sums[4][256];
  const int tid = threadIdx.x & 255, grp = threadIdx.x >> 8, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = tid >> 6, wm = wave % T::WM, wn = wave / T::WM;
  D* out = static_cast<D*>(a.out);
  const int tiles = a.mt * a.ntn;  // dh: by rows, then states; dW: by words, then states
  const int work = loss_join_blocks<T>(tiles), wg = blockIdx.y * gridDim.x + blockIdx.x;
  if (wg >= work + more.zero_wg) {
    if (wg < work + more.zero_wg + more.db_wg) sum_bias(more.db, wg - work - more.zero_wg, reinterpret_cast<float*>(sums));
    return;
  }
  if (wg >= work) {
    for (int n = wg - work; n < more.N; n += more.zero_wg)
      if (more.inv[n] < 0)
        for (int i = threadIdx.x; i < a.cols; i += 1024) out[(size_t)n * a.ld + i] = (D)0.f;
    return;
  }
  const int rows = a.is_dh ? *a.count : a.rows;
  const int q = wg & 3, unit = wg >> 2;
  const int tile = unit / (T::MB * T::NB), blk = unit % (T::MB * T::NB);
  const int m = blk / T::NB, n = blk % T::NB;
  const int mt = a.is_dh ? tile % a.mt : tile / a.ntn, nt = a.is_dh ? tile / a.mt : tile % a.ntn;
  if (nt * T::BN >= rows) return;
  const int row = nt * T::BN + wn * T::WTN + n * 32 + col;
  const size_t step = (size_t)tiles * (T::MB * T::NB) * 4 * 256;
  const float4* p = reinterpret_cast<const float4*>(a.part) + ((size_t)unit * 4 + q) * 256 + tid;
  float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4* from) {
#pragma unroll 8
    for (int k = grp; k < a.splits; k += 4) {
      const float4 v = from[k * step];
      r.x += v.x, r.y += v.y, r.z += v.z, r.w += v.w;
    }
  };
  if (row < rows) {
    add(p);
    if (a.two > 0) {  // the row's second pieces: row + two, in the same tile
      const int r2 = row + a.two, wn2 = r2 / T::WTN, n2 = r2 % T::WTN / 32;
      add(reinterpret_cast<const float4*>(a.part) + ((size_t)(tile * T::MB * T::NB + m * T::NB + n2) * 4 + q) * 256 +
          (wm + T::WM * wn2) * 64 + half * 32 + r2 % 32);
    }
  }
  if (a.splits > 1) {
    sums[grp][tid] = r;
    __syncthreads();
  }
  if (grp > 0) return;
  for (int k = 1; k < min(4, a.splits); ++k) {
    const float4 v = sums[k][tid];
    r.x += v.x, r.y += v.y, r.z += v.z, r.w += v.w;
  }
  const int c = mt * kLossM + wm * T::WTM + m * 32 + 8 * q + 4 * half;
  if (row >= rows) return;
  D* to = out + (size_t)(a.is_dh ? a.map[row] : row) * a.ld + c;
  typedef D D4 __attribute__((ext_vector_type(4)));
  if (c + 4 <= a.cols && (uintptr_t)to % sizeof(D4) == 0) {
    *reinterpret_cast<D4*>(to) = D4{(D)r.x, (D)r.y, (D)r.z, (D)r.w};
  } else {
    const float v[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < a.cols) to[j] = (D)v[j];
  }
}

template <int PASSES>
hipError_t launch_loss_dh_p(int BN, const LossGradArgs& a, hipStream_t st) {
  const dim3 gr(a.splits * (a.two > 0 ? 1 : loss_row_tiles(a.N, BN)) * a.mt), th(256);
  switch (BN) {
    case 256: loss_dh<LossT256, PASSES><<<gr, th, 0, st>>>(a); break;
    case 192: loss_dh<LossT192, PASSES><<<gr, th, 0, st>>>(a); break;
    case 128: loss_dh<LossT128, PASSES><<<gr, th, 0, st>>>(a); break;
    case 64: loss_dh<LossT64, PASSES><<<gr, th, 0, st>>>(a); break;
    default: loss_dh<LossT32, PASSES><<<gr, th, 0, st>>>(a); break;
  }
  return hipGetLastError();
}

template <int PASSES>
hipError_t launch_loss_dw_p(int BNh, const LossGradArgs& a, hipStream_t st) {
  const dim3 gr(a.grid), th(256);
  if constexpr (PASSES != 2) {  // dlogits in two pieces are those of at most 128 rows, whose state tiles are 64 wide
    if (BNh == 256) {
      loss_dw<LossT256, PASSES><<<gr, th, 0, st>>>(a);
      return hipGetLastError();
    }
    if (BNh == 128) {
      loss_dw<LossT128, PASSES><<<gr, th, 0, st>>>(a);
      return hipGetLastError();
    }
  } else if (BNh != 64) {
    return hipErrorInvalidValue;
  }
  loss_dw<LossT64, PASSES><<<gr, th, 0, st>>>(a);
  return hipGetLastError();
}

// row tiles of 192 or 256, state tiles of 256
template <int PASSES>
hipError_t launch_loss_both_p(int BN, const LossGradArgs& h, const LossGradArgs& w, hipStream_t st) {
  const dim3 gr(h.splits * loss_row_tiles(h.N, BN) * h.mt + w.splits * w.mt * w.ntn), th(256);
  if (BN == 192)
    loss_both<LossT192, LossT256, PASSES><<<gr, th, 0, st>>>(h, w);
  else
    loss_both<LossT256, LossT256, PASSES><<<gr, th, 0, st>>>(h, w);
  return hipGetLastError();
}

}  // namespace kb
