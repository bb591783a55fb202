// The losses of at most eight rows (of float32, scored: sixteen, in two turns): W is read once (twice for its gradient)
// and everything else is small, so the vector ALUs do, in float32 whatever the operands' type, and W needs no laying out,
// whatever its alignment.
//
// A workgroup takes chunks of 16 (few words: 8) x 16 bytes of words: threads of 16 bytes each along the words, and 16 or
// 32 slices along the states.  Forward: every thread sums its words' products over its slice's states for all rows, the
// states in LDS; the slices are summed through LDS; one wave a row takes the chunk into the row's running (max, sum),
// and threads pick the entries' logits.  Gradient: the same logits become dlogits in LDS, and a second walk over the
// states gives dW (a product over the rows, written as it comes) and the chunk's part of dh (summed over the threads
// along the words by halving what a lane keeps), which the workgroup adds up over its chunks in LDS.
//
// 8 rows of float32, 1,024 x 32,000: 55 us from memory (2.4 TB/s, one reading of W), 36 with W in the last-level cache; the
// gradients 77 (5.1 TB/s, three passes over its size, the second reading from that cache); 5 x 256 x 8,000 is bound by the
// launches (10 and 4 us of kernels; with gradients 35 in four).
#include <algorithm>
#include <type_traits>

#include "loss_load.hpp"
#include "loss_teacher.hpp"

namespace kb {

typedef __bf16 bf16x8f __attribute__((ext_vector_type(8)));

template <class S>
struct FewWords {
  static constexpr int N = 16 / sizeof(S);  // of a thread
};

// A thread's words of a row of W: by one load (of any alignment) where all of them exist (ALL), else the `left` ones.
template <bool ALL, class S>
__device__ __forceinline__ void few_load(const S* p, int left, float (&x)[FewWords<S>::N]) {
  constexpr int NW = FewWords<S>::N;
  if constexpr (!ALL) {
#pragma unroll
    for (int i = 0; i < NW; ++i) x[i] = i < left ? widen(p, i) : 0.f;
  } else {
    load16(p, x);
  }
}

template <bool ALL, class S>
__device__ __forceinline__ void few_store(S* p, int left, const float (&x)[FewWords<S>::N]) {
  constexpr int NW = FewWords<S>::N;
  if constexpr (sizeof(S) == 2) {
    bf16x8f r;
#pragma unroll
    for (int i = 0; i < NW; ++i) r[i] = (__bf16)x[i];
    if constexpr (ALL) {
      *reinterpret_cast<AnyU32x4*>(p) = __builtin_bit_cast(u32x4, r);
    } else {
#pragma unroll
      for (int i = 0; i < NW; ++i)
        if (i < left) reinterpret_cast<__bf16*>(p)[i] = r[i];
    }
  } else if constexpr (ALL) {
    *reinterpret_cast<AnyF32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
  } else {
#pragma unroll
    for (int i = 0; i < NW; ++i)
      if (i < left) p[i] = x[i];
  }
}

// v[0 .. NR) summed over TW lanes in a row, 16 or 8 (i: the lane among them); lane i gets the value that its bits name
// from the top, as many as NR needs, the same in the lanes that differ in the others.
template <int NR, int TW>
__device__ __forceinline__ float few_sum(float (&v)[NR], int i) {
  static_assert((TW == 16 || TW == 8) && NR <= 8, "at most eight values");
  auto step = [&](auto n_c, bool upper, auto move) {
    constexpr int n = decltype(n_c)::value;  // values kept before
    if constexpr (n > 1) {
#pragma unroll
      for (int r = 0; r < n / 2; ++r) {
        const float keep = upper ? v[r + n / 2] : v[r], give = upper ? v[r] : v[r + n / 2];
        v[r] = keep + move(give);
      }
    } else {
      v[0] += move(v[0]);
    }
  };
  auto half = [](int n) { return n > 1 ? n / 2 : 1; };
  constexpr int n3 = TW == 16 ? half(NR) : NR, n2 = half(n3), n1 = half(n2);
  if constexpr (TW == 16) step(std::integral_constant<int, NR>{}, (i & 8) != 0, [](float x) { return dpp_of<0x140>(x); });  // row_mirror
  step(std::integral_constant<int, n3>{}, (i & 4) != 0, [](float x) { return dpp_of<0x141>(x); });  // row_half_mirror
  step(std::integral_constant<int, n2>{}, (i & 2) != 0, [](float x) { return dpp_of<0x1b>(x); });   // quad_perm 3 2 1 0
  step(std::integral_constant<int, n1>{}, (i & 1) != 0, [](float x) { return dpp_of<0xb1>(x); });   // quad_perm 1 0 3 2
  return v[0];
}

// Floats of LDS that the states of nr rows take: whole 16 bytes, as what lies behind them asks.
__host__ __device__ inline size_t few_states(int H, int nr) { return ((size_t)H * nr + 3) / 4 * 4; }

template <class S, int NR, bool GRAD, int TW>
__global__ __launch_bounds__(256) void loss_few(LossFewArgs a) {
  constexpr int NW = FewWords<S>::N, CH = TW * NW, NS = 256 / TW;  // words of a chunk, slices
  extern __shared__ __align__(16) float dyn[];
  const size_t held = few_states(a.H, NR);
  // Eight rows' values of a state are read by 16 bytes; scored in float32, in pairs (8 x 1,024 x 32,000, W in the last-level
  // cache, a call: 40.8 us, by 16 bytes, with fewer registers and fewer loads under way, 42.7; bf16 and gradients are 1 to
  // 6% faster by 16 bytes).
  uint32_t first = 0;
  if constexpr (!GRAD && sizeof(S) == 4) asm("" : "+s"(first));  // the compiler does not know where they lie
  float* hs = dyn + first;                // H x NR states
  float* dhs = hs + held;                 // H x NR (gradient)
  float* red = dhs + (GRAD ? held : 0);   // 4 x NR x CH, written 16 bytes at a time
  float* xs = red + 4 * NR * CH;          // NR x CH logits, then dlogits
  float* rowv = xs + NR * CH;             // NR x 2: (lse, gradient)
  float* part = rowv + 2 * NR;                      // NR x K (gradient)
  int* tok = reinterpret_cast<int*>(part + (GRAD ? NR * a.K : 0));  // NR x K
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int ws = tid % TW, slice = tid / TW;
  const S* W = static_cast<const S*>(a.W);
  const S* h = static_cast<const S*>(a.h);
  const int N = a.N, H = a.H, V = a.V, K = a.K;

  // ---- rows and entries
  for (int n = wave; n < NR; n += 4) {
    bool any = false;
    if (n < N) {
      if (a.logit) {
        const TeacherRow r = teacher_row(a.token + n * K, a.logit + n * K, K, V, a.inv_t);
        any = r.any;
#pragma unroll
        for (int u = 0; u < 2; ++u)
          if (lane + 64 * u < K) {
            tok[n * K + lane + 64 * u] = r.token[u];
            if (GRAD) part[n * K + lane + 64 * u] = r.part[u];
          }
      } else {
        const int t = a.token[n];
        any = t >= 0 && t < V;
        if (lane == 0) {
          tok[n] = any ? t : -1;
          if (GRAD) part[n] = a.target_part;
        }
      }
    } else {
      for (int j = lane; j < K; j += 64) tok[n * K + j] = -1;
    }
    if (lane == 0) {
      rowv[2 * n] = any && GRAD ? a.lse[n] : INFINITY;
      rowv[2 * n + 1] = any ? (GRAD ? a.grad[n] * a.grad_scale : 1.f) : 0.f;  // forward: whether the row counts
    }
  }
  __syncthreads();
  for (int i = tid; i < H * NR; i += 256) {
    const int k = i / NR, n = i % NR;
    // rows left out are not read
    hs[i] = n < N && (GRAD ? rowv[2 * n] != INFINITY : rowv[2 * n + 1] != 0.f) ? widen(h, (size_t)n * H + k) : 0.f;
    if (GRAD) dhs[i] = 0.f;
  }
  __syncthreads();

  constexpr int RW = (NR + 3) / 4;  // rows of a wave
  float st_m[RW], st_s[RW], st_x[RW];
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    st_m[i] = kStatInit;
    st_s[i] = st_x[i] = 0.f;
  }
  const int chunks = (V + CH - 1) / CH;
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int v0 = c * CH, w0 = ws * NW, left = V - v0 - w0;
    const S* Wc = W + v0 + w0;
    // ---- logits: the slice's states
    float acc[NR][NW];
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int i = 0; i < NW; ++i) acc[n][i] = 0.f;
    auto take = [&](int k, const float (&w)[NW]) {
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const float x = hs[k * NR + n];
#pragma unroll
        for (int i = 0; i < NW; ++i) acc[n][i] = fmaf(x, w[i], acc[n][i]);
      }
    };
    if (left >= NW) {
      constexpr int U = 8;  // loads under way
      int k = slice;
      for (; k + NS * (U - 1) < H; k += NS * U) {
        float w[U][NW];
#pragma unroll
        for (int u = 0; u < U; ++u) few_load<true>(Wc + (size_t)(k + NS * u) * V, left, w[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) take(k + NS * u, w[u]);
      }
      for (; k < H; k += NS) {
        float w[NW];
        few_load<true>(Wc + (size_t)k * V, left, w);
        take(k, w);
      }
    } else if (left > 0) {
      for (int k = slice; k < H; k += NS) {
        float w[NW];
        few_load<false>(Wc + (size_t)k * V, left, w);
        take(k, w);
      }
    }
    // ---- over the slices: those of a wave, then the waves
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        if (TW == 8) acc[n][i] += dpp_of<0x128>(acc[n][i]);  // row_ror by 8
        acc[n][i] += __shfl_xor(acc[n][i], 16, 64);
        acc[n][i] += __shfl_xor(acc[n][i], 32, 64);
      }
      if (lane < TW) {
#pragma unroll
        for (int i = 0; i < NW; i += 4)
          *reinterpret_cast<float4*>(&red[(wave * NR + n) * CH + w0 + i]) =
              make_float4(acc[n][i], acc[n][i + 1], acc[n][i + 2], acc[n][i + 3]);
      }
    }
    __syncthreads();
    for (int i = tid; i < NR * CH; i += 256) {
      const int n = i / CH, w = i % CH;
      float x = -INFINITY;
      if (v0 + w < V) x = ((red[i] + red[NR * CH + i]) + (red[2 * NR * CH + i] + red[3 * NR * CH + i])) + a.b[v0 + w];
      if constexpr (GRAD) {
        const float p = exp2_fast(fmaf(x, a.inv_t, -rowv[2 * n]) * kL2E), g = rowv[2 * n + 1];
        x = v0 + w < V ? g * (p - a.rest) : 0.f;
      }
      xs[i] = x;
    }
    __syncthreads();
    // ---- entries: each of a row is of another word
    for (int e = tid; e < NR * K; e += 256) {
      const int t = tok[e] - v0;
      if (tok[e] >= 0 && t >= 0 && t < CH) {
        const int n = e / K;
        if constexpr (GRAD)
          xs[n * CH + t] = fmaf(-rowv[2 * n + 1], part[e], xs[n * CH + t]);
        else
          a.xt[e] = xs[n * CH + t];
      }
    }
    if constexpr (!GRAD) {
#pragma unroll
      for (int i = 0; i < RW; ++i) {
        const int n = wave + 4 * i;
        if (n >= NR) continue;
        constexpr int NU = (CH + 63) / 64;
        float x[NU], m = st_m[i];
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          x[u] = CH >= 64 || lane < CH ? xs[n * CH + u * 64 + lane] : -INFINITY;
          m = fmaxf(m, x[u]);
        }
        float s = st_s[i] * exp2_fast((st_m[i] - m) * (kL2E * a.inv_t));
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          s += exp2_fast((x[u] - m) * (kL2E * a.inv_t));
          if ((CH >= 64 || lane < CH) && v0 + u * 64 + lane < V) st_x[i] += x[u];
        }
        st_m[i] = m;
        st_s[i] = s;
      }
      __syncthreads();  // xs is written again
    } else {
      __syncthreads();
      if (a.db)
        for (int w = tid; w < CH; w += 256)
          if (v0 + w < V) {
            float s = 0.f;
#pragma unroll
            for (int n = 0; n < NR; ++n) s += xs[n * CH + w];
            a.db[v0 + w] = s;
          }
      if (a.dW || a.dh_part) {
        float g[NR][NW];
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int i = 0; i < NW; ++i) g[n][i] = xs[n * CH + w0 + i];
        auto walk = [&](auto all, auto wants_w, auto wants_h) {
          constexpr bool ALL = decltype(all)::value, DW = decltype(wants_w)::value, DH = decltype(wants_h)::value;
          constexpr int U = 4;
          auto turn = [&](int k, const float (&w)[NW]) {
            if constexpr (DW) {
              float d[NW];
#pragma unroll
              for (int i = 0; i < NW; ++i) d[i] = 0.f;
#pragma unroll
              for (int n = 0; n < NR; ++n) {
                const float x = hs[k * NR + n];
#pragma unroll
                for (int i = 0; i < NW; ++i) d[i] = fmaf(x, g[n][i], d[i]);
              }
              few_store<ALL>(static_cast<S*>(a.dW) + (size_t)k * V + v0 + w0, left, d);
            }
            if constexpr (DH) {
              float v[NR];
#pragma unroll
              for (int n = 0; n < NR; ++n) {
                v[n] = 0.f;
#pragma unroll
                for (int i = 0; i < NW; ++i) v[n] = fmaf(g[n][i], w[i], v[n]);
              }
              const float s = few_sum<NR, TW>(v, ws);
              constexpr int SAME = TW / NR;  // lanes that have the same value
              if (ws % SAME == 0) dhs[k * NR + ws / SAME] += s;
            }
          };
          int k = slice;
          if constexpr (ALL) {
            for (; k + NS * (U - 1) < H; k += NS * U) {
              float w[U][NW];
              if constexpr (DH) {
#pragma unroll
                for (int u = 0; u < U; ++u) few_load<true>(Wc + (size_t)(k + NS * u) * V, left, w[u]);
              }
#pragma unroll
              for (int u = 0; u < U; ++u) turn(k + NS * u, w[u]);
            }
          }
          for (; k < H; k += NS) {
            float w[NW];
            if constexpr (DH) few_load<ALL>(Wc + (size_t)k * V, left, w);
            turn(k, w);
          }
        };
        using Y = std::true_type;
        using No = std::false_type;
        // the sums over lanes are all lanes' work: one that has no words, or not all, takes its whole wave along
        if (__builtin_amdgcn_ballot_w64(left < NW) == 0ull) {
          if (a.dW && a.dh_part)
            walk(Y{}, Y{}, Y{});
          else if (a.dW)
            walk(Y{}, Y{}, No{});
          else
            walk(Y{}, No{}, Y{});
        } else if (a.dW && a.dh_part) {
          walk(No{}, Y{}, Y{});
        } else if (a.dW) {
          walk(No{}, Y{}, No{});
        } else {
          walk(No{}, No{}, Y{});
        }
      }
      __syncthreads();
    }
  }
  if constexpr (GRAD) {
    if (a.dh_part)
      for (int i = tid; i < H * NR; i += 256) a.dh_part[(size_t)blockIdx.x * H * NR + i] = dhs[i];
  } else {
#pragma unroll
    for (int i = 0; i < RW; ++i) {
      const int n = wave + 4 * i;
      float m = st_m[i], s = st_s[i], x = st_x[i];
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) {
        const float mo = __shfl_xor(m, d, 64), so = __shfl_xor(s, d, 64);
        const float mm = fmaxf(m, mo);
        s = s * exp2_fast((m - mm) * (kL2E * a.inv_t)) + so * exp2_fast((mo - mm) * (kL2E * a.inv_t));
        m = mm;
        x += __shfl_xor(x, d, 64);
      }
      if (lane == 0 && n < N) {
        a.stat[(size_t)n * gridDim.x + blockIdx.x] = make_float2(m, s);
        a.sumx[(size_t)n * gridDim.x + blockIdx.x] = x;
      }
    }
  }
}

// loss and log-sum-exp, a wave each row.
__global__ __launch_bounds__(64) void loss_few_finish(LossFewArgs a) {
  const int lane = threadIdx.x, n = blockIdx.x, K = a.K;
  float known = 0.f;
  bool any;
  int tok[2] = {-1, -1};
  float part[2] = {0.f, 0.f};
  if (a.logit) {
    const TeacherRow r = teacher_row(a.token + n * K, a.logit + n * K, K, a.V, a.inv_t);
    any = r.any;
    known = r.known;
#pragma unroll
    for (int u = 0; u < 2; ++u) tok[u] = r.token[u], part[u] = r.part[u];
  } else {
    const int t = a.token[n];
    any = t >= 0 && t < a.V;
    if (lane == 0 && any) tok[0] = t, part[0] = a.target_part;
  }
  if (!any) {
    if (lane == 0) a.loss[n] = a.lse_out[n] = 0.f;
    return;
  }
  const float c = kL2E * a.inv_t;
  float M = kStatInit, S = 0.f, X = 0.f;
  for (int i = lane; i < a.grid; i += 64) {
    const float2 v = a.stat[(size_t)n * a.grid + i];
    const float m = fmaxf(M, v.x);
    S = S * exp2f((M - m) * c) + v.y * exp2f((v.x - m) * c);
    M = m;
    X += a.sumx[(size_t)n * a.grid + i];
  }
  float dot = 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (tok[u] >= 0 && part[u] != 0.f) dot += part[u] * a.xt[n * K + lane + 64 * u];  // of no weight: also where x = -inf
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float mo = __shfl_xor(M, d, 64), so = __shfl_xor(S, d, 64);
    X += __shfl_xor(X, d, 64);
    dot += __shfl_xor(dot, d, 64);
    const float m = fmaxf(M, mo);
    S = S * exp2f((M - m) * c) + so * exp2f((mo - m) * c);
    M = m;
  }
  if (lane == 0) {
    const float lse = M * a.inv_t + logf(S);
    float l = lse - dot * a.inv_t + known;
    if (a.rest != 0.f) l -= a.rest * X;
    a.loss[n] = l * a.t2;
    a.lse_out[n] = lse;
  }
}

// dh from the workgroups' parts: 32 groups of threads take every 32nd part of 32 values each, in order.
template <class D>
__global__ __launch_bounds__(1024) void loss_few_join(LossFewArgs a, int held) {
  __shared__ float sums[32][33];
  const int x = threadIdx.x & 31, grp = threadIdx.x >> 5;
  const int i = blockIdx.x * 32 + x, total = a.H * held;
  float s = 0.f;
  if (i < total) {
#pragma unroll 8
    for (int p = grp; p < a.grid; p += 32) s += a.dh_part[(size_t)p * total + i];
  }
  sums[grp][x] = s;
  __syncthreads();
  if (grp == 0 && i < total) {
    float t = 0.f;
#pragma unroll
    for (int g = 0; g < 32; ++g) t += sums[g][x];
    const int k = i / held, n = i % held;
    if (n < a.N) static_cast<D*>(a.dh)[(size_t)n * a.H + k] = (D)t;
  }
}

int few_held(int N) { return N <= 1 ? 1 : N <= 2 ? 2 : N <= 4 ? 4 : 8; }

// Threads along the words: 8 where chunks of 16 would leave half of the card idle (bf16, 8 x 512 x 8,000 with gradients:
// 42 us, 77 in chunks of 16; 8 x 512 x 32,000: 60 in both, one row 45 and 38).
static int few_threads(bool bf16, int V) { return V <= 128 * 16 * (bf16 ? 8 : 4) ? 8 : 16; }

static size_t few_lds(bool bf16, bool grad, int N, int H, int K, int threads) {
  const size_t nr = few_held(N), ch = threads * (bf16 ? 8 : 4);
  return (few_states(H, nr) * (grad ? 2 : 1) + 5 * nr * ch + 2 * nr + nr * K * (grad ? 2 : 1)) * 4;
}

// bf16 rows of a large W are the matrix cores' (8 x 1,024 x 32,000: 24 us there and 35 here, with gradients 87 and 97; one
// row of 1,024 x 60,000 33 and 31, 140 and 168; 8 x 512 x 32,000 21 and 23, 71 and 60).  Those of float32 are not: W would
// have to be laid out in pieces (8 x 1,024 x 60,000: 275 us there, 80 here).
bool few_fits(bool bf16, int N, int H, int V) {
  if (N > kFewRows || few_lds(true, true, N, H, kLossMaxK, 16) > 150 * 1024) return false;
  return !bf16 || (long long)H * V * (N + 4) <= 1ll << 28;
}

int few_grid(bool bf16, int V) {
  const int ch = few_threads(bf16, V) * (bf16 ? 8 : 4);
  return std::min((V + ch - 1) / ch, kFewGrid);
}

template <class S, bool GRAD, int TW>
static hipError_t few_launch(const LossFewArgs& a, size_t lds, hipStream_t st) {
  const dim3 gr(a.grid), th(256);
  void (*f)(LossFewArgs) = nullptr;
  switch (few_held(a.N)) {
    case 1: f = loss_few<S, 1, GRAD, TW>; break;
    case 2: f = loss_few<S, 2, GRAD, TW>; break;
    case 4: f = loss_few<S, 4, GRAD, TW>; break;
    default: f = loss_few<S, 8, GRAD, TW>; break;
  }
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  f<<<gr, th, lds, st>>>(a);
  return hipGetLastError();
}

template <class S>
static hipError_t few_launch(bool grad, int threads, const LossFewArgs& a, size_t lds, hipStream_t st) {
  if (threads == 16) return grad ? few_launch<S, true, 16>(a, lds, st) : few_launch<S, false, 16>(a, lds, st);
  return grad ? few_launch<S, true, 8>(a, lds, st) : few_launch<S, false, 8>(a, lds, st);
}

hipError_t launch_loss_few(bool bf16, bool grad, const LossFewArgs& a, hipStream_t st) {
  const int threads = few_threads(bf16, a.V);
  const size_t lds = few_lds(bf16, grad, a.N, a.H, a.K, threads);
  return bf16 ? few_launch<uint16_t>(grad, threads, a, lds, st) : few_launch<float>(grad, threads, a, lds, st);
}

hipError_t launch_loss_few_finish(const LossFewArgs& a, hipStream_t st) {
  loss_few_finish<<<dim3(a.N), dim3(64), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_loss_few_join(bool bf16, const LossFewArgs& a, hipStream_t st) {
  const int held = few_held(a.N);
  const dim3 gr((a.H * held + 31) / 32), th(1024);
  if (bf16)
    loss_few_join<__bf16><<<gr, th, 0, st>>>(a, held);
  else
    loss_few_join<float><<<gr, th, 0, st>>>(a, held);
  return hipGetLastError();
}

}  // namespace kb
