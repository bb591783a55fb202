// The matrix products of the output layer's losses, on the bf16 matrix cores.
//
// C[m, n] = sum_k A[m, k] B[n, k] in tiles of 256 x BN by four waves, in stages of 32 steps of k.  Each side is in
// memory either along k ("along": a row of k after the other) or across it (all m of one k, then the next); the
// three products of a loss need every pairing but one:
//
//   logits   A = W (words across states),  B = h (along the states)
//   dh       A = W (along the words),      B = dlogits (along the words)
//   dW       A = dlogits (across rows),    B = h (across rows)
//
// so nothing is transposed in memory.  A stage of either kind takes 64 bytes of every row or column of the tile and
// reaches LDS by the global->LDS DMA, three stages ahead, in a ring of four.  Along k, rows lie as 64-byte slices
// and a fragment is one 16-byte read; across k, as 32 runs of the tile's width, and a fragment is two transposing
// reads (ds_read_b64_tr_b16).  Both are XOR-swizzled in 16-byte chunks, by the addresses of the loads, so that
// fragment reads meet distinct banks.
//
// Between a stage's two halves of 16 steps stands its only barrier: the first half's products run while the second
// half's fragments are read, the second half's while the next stage's first are; the DMA of the stage three ahead
// goes into the buffer that all waves have left before the barrier of the stage before.  The ring runs on over a
// workgroup's tiles: the next tile's first three stages arrive while a tile's epilogue works, which may use the
// buffer of the tile's last stage.
//
// float32 operands come as three bf16 pieces each (planes; 8 + 8 + 8 significand bits), and k runs six times: over
// the products of weight 1 to 2^-16.  The three left out are below 2^-24 of the product together.
#pragma once

#include "k1_common.hpp"
#include "loss_common.hpp"

namespace kb {

// One side of a product. Strided: element (x, k) at p[k * ld + x0 + x]; else p[(x0 + x) * ld + k].
struct MmSide {
  const uint16_t* p;
  int ld;
  size_t plane;   // values from one bf16 piece to the next
  int lim;        // CLAMP only. Strided: columns there are from x0 on; else rows there are from x0 on
  int klim;       // CLAMP, not strided: steps of k there are
};

__device__ __forceinline__ const void* uniform_ptr(const void* x) {
  const uint64_t p = reinterpret_cast<uint64_t>(x);
  return reinterpret_cast<const void*>(((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(p >> 32)) << 32) |
                                       (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)p));
}

// One DMA instruction: lane i's 16 bytes from base + voff to LDS byte lds + PLUS + 16 i.  The load needs five wait
// states after a VALU instruction that wrote its base: NOP 0 where the compiler keeps the base in scalar registers (the
// build checks that; isa_check.py), 4 where it may come from a vector register.
template <int PLUS, int NOP>
__device__ __forceinline__ void dma16_at(uint32_t voff, const void* sbase, uint32_t lds) {
  asm volatile("s_add_i32 m0, %2, %3\n\ts_nop %4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff),
               "s"(uniform_ptr(sbase)), "s"(__builtin_amdgcn_readfirstlane(lds)), "i"(PLUS), "i"(NOP)
               : "m0", "scc");
}

// A kernel's arguments, read anew wherever this is called: what only a tile's start or end needs does not take scalar
// registers in the main loop (which otherwise spills the DMA's addresses).
template <class Args>
__device__ __forceinline__ const __attribute__((address_space(4))) Args* args_again() {
  auto p = (const __attribute__((address_space(4))) Args*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}

__device__ __forceinline__ void in_acc(f32x16& x) { asm volatile("" : "+a"(x)); }

template <int R>
struct MmGeom {
  static constexpr int BYTES = R * 2 * kLossStage;
  static constexpr int ALL = BYTES / 1024;             // DMA instructions a stage
  static constexpr int OPS = ALL >= 4 ? ALL / 4 : 1;   // of each wave (fewer than four: some do the same one)
};

// Which pieces of A and B a pass multiplies, two bits a pass.
template <int PASSES_, uint32_t A_, uint32_t B_>
struct MmPasses {
  static constexpr int N = PASSES_;
  static constexpr uint32_t A = A_, B = B_;
};
using MmOne = MmPasses<1, 0, 0>;
using MmTwoA = MmPasses<2, 0u | 1u << 2, 0>;  // A in two pieces
// float32: (0,0) (0,1) (1,0) (1,1) (0,2) (2,0)
using MmSix = MmPasses<6, 0u | 0u << 2 | 1u << 4 | 1u << 6 | 0u << 8 | 2u << 10,
                       0u | 1u << 2 | 0u << 4 | 1u << 6 | 2u << 8 | 0u << 10>;

template <int BASE, int NOP>
__device__ __forceinline__ void dma_i(const uint32_t* off, int i, const void* src, uint32_t lds) {
  switch (i) {
    case 0: dma16_at<BASE, NOP>(off[0], src, lds); break;
    case 1: dma16_at<BASE + 1 * 1024, NOP>(off[1], src, lds); break;
    case 2: dma16_at<BASE + 2 * 1024, NOP>(off[2], src, lds); break;
    default: dma16_at<BASE + 3 * 1024, NOP>(off[3], src, lds); break;
  }
}

// T: tile; AS, BS: the side is strided; AC: side A is clamped to its limits; PS: MmPasses.
// STORES: vector memory instructions that every wave issues in each epilogue, at least: the loads of the two stages
// after it were issued before them, and are not waited for as if they came after (the counter is in order).
// nt tiles of nk stages a pass.  tile(t, A, B): the sides of tile t; init(t, acc); epi(t, acc, lds): lds is a stage's
// buffer that is free until epi returns.
template <class T, bool AS, bool BS, bool AC, class PS, int STORES, class TileFn, class InitFn, class EpiFn>
__device__ __forceinline__ void mm_run(uint32_t ring, int nt_, int nk_, TileFn tile, InitFn init, EpiFn epi) {
  const int nt = __builtin_amdgcn_readfirstlane(nt_), nk = __builtin_amdgcn_readfirstlane(nk_);
  constexpr int MB = T::MB, NB = T::NB, BM = T::BM, BN = T::BN, PASSES = PS::N;
  constexpr int NOP = PASSES > 1 ? 4 : 0;  // several passes: the compiler selects the bases in vector registers
  using GA = MmGeom<BM>;
  using GB = MmGeom<BN>;
  constexpr int STAGE = GA::BYTES + GB::BYTES;
  constexpr int OPS = GA::OPS + GB::OPS;
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
  const int total = nt * nk * PASSES;

  // ---- what is loaded
  MmSide A, B;
  uint32_t aload[GA::OPS], bload[GB::OPS];  // byte offsets from the stage's first element
  const char *asrc = nullptr, *bsrc = nullptr;
  uint32_t astep = 0, bstep = 0;  // bytes from a stage to the next
  int t_issue = 0, k_issue = 0, pass = 0, issued = 0;

  // offsets of a clamped side along k count from this many steps before the stage: they are never negative
  constexpr int kBack = AC && !AS ? 512 : 0;
  auto offsets = [&](auto strided, auto r_c, auto clamp, const MmSide& s, int k0, uint32_t* off) {
    constexpr bool S = decltype(strided)::value;
    constexpr int R = decltype(r_c)::value;
    using G = MmGeom<R>;
#pragma unroll
    for (int i = 0; i < G::OPS; ++i) {
      const int q = G::ALL >= 4 ? wave * G::OPS + i : (wave & (G::ALL - 1));
      const int slot = q * 64 + lane;
      if constexpr (S) {
        const int r = slot / (R / 8);
        int c = ((slot % (R / 8)) ^ (wswz(r) & (R / 8 - 1))) * 8;
        if constexpr (decltype(clamp)::value) c = min(c, s.lim - 8);
        off[i] = (uint32_t)r * (uint32_t)s.ld * 2u + (uint32_t)c * 2u;
      } else {
        int n = slot >> 2;
        int c = ((slot & 3) ^ hswz(n)) * 8;
        if constexpr (decltype(clamp)::value) {
          n = min(n, s.lim - 1);
          c = min(k0 + c, s.klim - 8) - k0;  // negative past the end, where less than kBack steps are filled up
          off[i] = (uint32_t)n * (uint32_t)s.ld * 2u + (uint32_t)(c + kBack) * 2u;
        } else {
          off[i] = (uint32_t)n * (uint32_t)s.ld * 2u + (uint32_t)c * 2u;
        }
      }
    }
  };
  using SA = std::integral_constant<bool, AS>;
  using SB = std::integral_constant<bool, BS>;
  using CA = std::integral_constant<bool, AC>;
  using CB = std::false_type;
  using RA = std::integral_constant<int, BM>;
  using RB = std::integral_constant<int, BN>;
  auto sources = [&]() {
    asrc = reinterpret_cast<const char*>(A.p);
    bsrc = reinterpret_cast<const char*>(B.p);
    if constexpr (PASSES > 1) {
      asrc += (size_t)((PS::A >> (2 * pass)) & 3u) * A.plane * 2;
      bsrc += (size_t)((PS::B >> (2 * pass)) & 3u) * B.plane * 2;
    }
    asrc = static_cast<const char*>(uniform_ptr(asrc));
    bsrc = static_cast<const char*>(uniform_ptr(bsrc));
    asm volatile("s_nop 4");  // whatever VALU instruction wrote these registers last: five states before the DMA
  };
  auto tile_sources = [&]() {
    tile(t_issue, A, B);
    astep = AS ? (uint32_t)__builtin_amdgcn_readfirstlane(kLossStage * 2 * A.ld) : kLossStage * 2;
    bstep = BS ? (uint32_t)__builtin_amdgcn_readfirstlane(kLossStage * 2 * B.ld) : kLossStage * 2;
    offsets(SA{}, RA{}, CA{}, A, 0, aload);
    offsets(SB{}, RB{}, CB{}, B, 0, bload);
    sources();
  };
  // a wave's first DMA instruction of each side
  const uint32_t wave_a = (GA::ALL >= 4 ? wave * GA::OPS : (wave & (GA::ALL - 1))) * 1024;
  const uint32_t wave_b = (GB::ALL >= 4 ? wave * GB::OPS : (wave & (GB::ALL - 1))) * 1024;
  auto issue_a = [&](uint32_t buf, int i) {
    if (i == 0 && AC && !AS) {
      // the stage that reaches the end of k has offsets of its own
      if ((k_issue + 1) * kLossStage > A.klim) offsets(SA{}, RA{}, CA{}, A, k_issue * kLossStage, aload);
    }
    dma_i<0, NOP>(aload, i, asrc - kBack * 2, buf + wave_a);
  };
  auto issue_b = [&](uint32_t buf, int i) {
    dma_i<GA::BYTES, NOP>(bload, i, bsrc, buf + wave_b);
  };
  auto issue_done = [&]() {
    ++issued;
    ++k_issue;
    asrc += astep;
    bsrc += bstep;
    if (k_issue == nk) {
      k_issue = 0;
      ++pass;
      if (PASSES > 1 && pass < PASSES) {
        sources();
        if (AC && !AS) offsets(SA{}, RA{}, CA{}, A, 0, aload);
      } else {
        pass = 0;
        ++t_issue;
        if (t_issue < nt) tile_sources();
      }
    }
  };
  auto issue_stage = [&](uint32_t buf) {
#pragma unroll
    for (int i = 0; i < GA::OPS; ++i) issue_a(buf, i);
#pragma unroll
    for (int i = 0; i < GB::OPS; ++i) issue_b(buf, i);
    issue_done();
  };

  // ---- fragments
  struct Frag {
    bf16x8 a[MB], b[NB];
  };
  uint32_t afrag[AS ? MB : 2], bfrag[BS ? NB : 2];
  auto frag_offsets = [&](auto strided, auto r_c, int w0, uint32_t base, uint32_t* off, int nblk) {
    constexpr bool S = decltype(strided)::value;
    constexpr int R = decltype(r_c)::value;
    if constexpr (S) {
      const int g = lane >> 4, j = lane & 15;
      const int r0 = 8 * (g >> 1) + (j >> 2);
#pragma unroll
      for (int x = 0; x < nblk; ++x) {
        const int c = w0 + x * 32 + 16 * (g & 1) + 4 * (j & 3);
        off[x] = base + (uint32_t)(r0 * R + (((c >> 3) ^ (wswz(r0) & (R / 8 - 1))) << 3) + (c & 7)) * 2u;
      }
    } else {
      const int n = w0 + col;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) off[kk] = base + (uint32_t)(n * 64 + (((kk * 2 + half) ^ hswz(n)) * 16));
    }
  };
  frag_offsets(SA{}, RA{}, wm * T::WTM, 0u, afrag, MB);
  frag_offsets(SB{}, RB{}, wn * T::WTN, (uint32_t)GA::BYTES, bfrag, NB);
  auto rd_side = [&](auto strided, auto r_c, uint32_t buf, const uint32_t* off, int kk, int x) -> bf16x8 {
    constexpr bool S = decltype(strided)::value;
    constexpr int R = decltype(r_c)::value;
    if constexpr (S) {
      const uint32_t at = buf + off[x] + kk * 16 * R * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KB_LDS s16x4*)(uintptr_t)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KB_LDS s16x4*)(uintptr_t)(at + 4 * R * 2));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *(const KB_LDS bf16x8*)(uintptr_t)(buf + off[kk] + x * 2048);
    }
  };
  // fragment u of a set in the order in which the products need them: a0, all b, the other a
  constexpr int NF = MB + NB;
  auto rd = [&](uint32_t buf, int kk, int u, Frag& f) {
    if (u == 0)
      f.a[0] = rd_side(SA{}, RA{}, buf, afrag, kk, 0);
    else if (u <= NB)
      f.b[u - 1] = rd_side(SB{}, RB{}, buf, bfrag, kk, u - 1);
    else
      f.a[u - NB] = rd_side(SA{}, RA{}, buf, afrag, kk, u - NB);
  };
  f32x16 acc[MB][NB];
  auto mf = [&](const Frag& f, int i) {
    const int m = i / NB, n = i % NB;
    acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[m], f.b[n], acc[m][n], 0, 0, 0);
  };
  constexpr int NM = MB * NB;
  // the product after which fragment u of the next half is read (in eighths of a product), and DMA i issued
  auto frag_slot = [](int u, int eighths) { return u * eighths * NM / (8 * 16) < NM ? u * eighths * NM / (8 * 16) : NM - 1; };
  auto slot_of = [](int i, int n) { return NM >= 8 ? NM / n * i + NM / n - 1 : (i < NM ? i : NM - 1); };
  constexpr int SP1 = 12 * 8 / NF, SP0 = 16 * 8 / NF;

  Frag F0, F1;
  if (total > 0) {
    tile_sources();
#pragma unroll
    for (int s = 0; s < 3; ++s)
      if (issued < total) issue_stage(ring + s * STAGE);
    if (total >= 3)
      wait_vm<2 * OPS>();
    else if (total == 2)
      wait_vm<OPS>();
    else
      wait_vm<0>();
    lds_barrier();
  }

  int g = 0, after_epi = 0;
  auto body = [&](auto rc) {
    constexpr bool read_next = decltype(rc)::value;
    const uint32_t cur = ring + (uint32_t)(g & 3) * STAGE;
    const uint32_t nxt = ring + (uint32_t)((g + 1) & 3) * STAGE;
    const uint32_t fill = ring + (uint32_t)((g + 3) & 3) * STAGE;
    const bool more = issued < total;
#pragma unroll
    for (int i = 0; i < NM; ++i) {
      mf(F0, i);
#pragma unroll
      for (int u = 0; u < NF; ++u)
        if (frag_slot(u, SP1) == i) rd(cur, 1, u, F1);
      if (more) {
#pragma unroll
        for (int o = 0; o < GA::OPS; ++o)
          if (slot_of(o, GA::OPS) == i) issue_a(fill, o);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // stage g + 1 has landed when no more than what was issued after it is under way
    constexpr int LATER = OPS + GA::OPS + STORES < 63 ? STORES : 63 - OPS - GA::OPS;
    if (g + 3 < total && STORES > 0 && after_epi > 0)
      wait_vm<OPS + GA::OPS + LATER>();
    else if (g + 3 < total)
      wait_vm<OPS + GA::OPS>();
    else if (g + 2 < total)
      wait_vm<OPS>();
    else
      wait_vm<0>();
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NM; ++i) {
      mf(F1, i);
      if constexpr (read_next) {
#pragma unroll
        for (int u = 0; u < NF; ++u)
          if (frag_slot(u, SP0) == i) rd(nxt, 0, u, F0);
      }
      if (more) {
#pragma unroll
        for (int o = 0; o < GB::OPS; ++o)
          if (slot_of(o, GB::OPS) == i) issue_b(fill, o);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (more) issue_done();
    ++g;
    --after_epi;
  };
  for (int t = 0; t < nt; ++t) {
    init(t, acc);
    if (nk > 0) {
      const uint32_t first = ring + (uint32_t)(g & 3) * STAGE;
#pragma unroll
      for (int u = 0; u < NF; ++u) rd(first, 0, u, F0);
      for (int s = 1; s < nk * PASSES; ++s) body(std::true_type{});
      body(std::false_type{});
    }
    epi(t, acc, ring + (uint32_t)((g + 3) & 3) * STAGE);
    after_epi = 2;
    if (t + 1 < nt) lds_barrier();  // the next stage's DMA goes into the buffer that the epilogue had
  }
}

}  // namespace kb
