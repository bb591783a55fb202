// Rotary positions and the append of new tokens to the attention cache.
//
// A pair (x, y) of a head turned by the angle a = pos * freq: (x cos a - y sin a,
// x sin a + y cos a), times the amplitude.
//
// Few operations a byte: what bounds it is the stream of rows in and out, and for a step's few
// rows the chain launch, position, angle, store.  A workgroup takes one row.  Its threads work out
// each angle once into LDS (the heads share them) while the row's values are on their way, then
// turn or copy them in pieces of V values, 16 bytes where every row starts at 16 bytes and the
// turned part is whole pairs of pieces, else one value.
//
// Kernel time, the least of 20: 8,200 tokens of 32 + 8 + 8 heads of 128 bf16 values 37.0 us, 202 MB in and out
// at 5.5 TB/s (a large copy: 4.8 to 5.2); 5 tokens 3.3 us.
#include "cache_common.hpp"
#include "cache_slot.hpp"

namespace kb {

// cos and sin of pos * freq times the amplitude.  The angle is reduced in 64
// bits: at position 10^6 a float32 product is off by up to 0.03 radians.
__device__ __forceinline__ float2 turn_of(int pos, double freq, float amplitude) {
  const double quarters = (double)pos * freq * 0.63661977236758134308;  // 2 / pi
  const double whole = rint(quarters);
  float s, c;
  sincospif(0.5f * (float)(quarters - whole), &s, &c);
  const int n = (int)((long long)whole & 3);
  const float cs = (n & 1) ? s : c, sn = (n & 1) ? c : s;
  return make_float2(((n + 1) & 2) ? -amplitude * cs : amplitude * cs, (n & 2) ? -amplitude * sn : amplitude * sn);
}

constexpr int kAppendT = 256;

template <class T, int V, bool PAIRS>
__global__ __launch_bounds__(kAppendT) void cache_append_rows(AppendArgs a) {
  struct Piece {
    T x[V];
  };
  __shared__ float2 turn[kCacheMaxDim / 2];
  const int r = blockIdx.x, tid = threadIdx.x;
  if (r >= rows_of(a.R, a.n_dev)) return;
  const CacheView& c = a.c;
  const int D = c.dim, half = a.rot / 2, H = a.q_heads + c.heads;
  const int s = cache_seq(c, a.seq, r);
  const int len = a.length[r];
  const int pos = a.pos ? a.pos[r] : (int)(uint32_t(len) - 1u);  // (stored only where there is a slot)
  int slot = s < 0 ? -1 : new_slot(len, c.cap);
  int64_t row = 0;
  if (slot >= 0) {
    row = cache_row(c, c.table + (int64_t)s * c.max_pages, 0, slot);
    if (row < 0) slot = -1;
  }
  // head h of queries, then of keys: where it comes from and goes to (null: nowhere)
  const int Q = a.q_heads, log_ps = c.log_ps;
  const T *q = (const T*)a.q + r * a.q_stride, *k = (const T*)a.k_new + r * a.k_stride,
          *v = (const T*)a.v_new + r * a.v_stride;
  T *q_out = (T*)a.q_out + (int64_t)r * Q * D, *k_out = slot < 0 ? nullptr : (T*)c.k + row * D,
    *v_out = (T*)c.v + row * D;
  auto from = [=](int h) { return h < Q ? q + (int64_t)h * D : k + (int64_t)(h - Q) * D; };
  auto to = [=](int h) {
    return h < Q ? q_out + (int64_t)h * D : k_out ? k_out + ((int64_t)(h - Q) << log_ps) * D : nullptr;
  };
  auto load = [](const T* p) {
    Piece x;
    __builtin_memcpy(&x, __builtin_assume_aligned(p, sizeof(Piece)), sizeof(Piece));
    return x;
  };
  auto store = [](T* p, const Piece& x) {
    __builtin_memcpy(__builtin_assume_aligned(p, sizeof(Piece)), &x, sizeof(Piece));
  };

  // a turned item: V pairs, in two pieces that lie half the turned part apart or side by side
  const int per = half / V, turned = H * per;
  auto place = [=](int i, int& h, int& u, int& lo, int& hi) {
    h = i / per;
    u = i - h * per;
    lo = PAIRS ? 2 * V * u : V * u;
    hi = PAIRS ? lo + V : lo + half;
  };
  constexpr int N = V > 1 ? 4 : 8;  // items in flight a thread
  for (int i0 = 0; i0 < turned || i0 == 0; i0 += N * kAppendT) {
    Piece x[N], y[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = i0 + j * kAppendT + tid;
      int h, u, lo, hi;
      if (i < turned) {
        place(i, h, u, lo, hi);
        x[j] = load(from(h) + lo);
        y[j] = load(from(h) + hi);
      }
    }
    if (i0 == 0) {
      if (tid < half) turn[tid] = turn_of(pos, a.freq[tid], a.amplitude);
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = i0 + j * kAppendT + tid;
      int h, u, lo, hi;
      if (i < turned) {
        place(i, h, u, lo, hi);
        T* out = to(h);
        Piece both[2] = {x[j], y[j]}, res[2];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          // pair V u + e: values e of both pieces, or 2e and 2e + 1 of the two in sequence
          const float2 cs = turn[V * u + e];
          const int pa = PAIRS ? 2 * e : e, pb = PAIRS ? 2 * e + 1 : V + e;
          const float f = (float)both[pa / V].x[pa % V], w = (float)both[pb / V].x[pb % V];
          res[pa / V].x[pa % V] = (T)(f * cs.x - w * cs.y);
          res[pb / V].x[pb % V] = (T)(f * cs.y + w * cs.x);
        }
        if (out) {
          store(out + lo, res[0]);
          store(out + hi, res[1]);
        }
      }
    }
  }
  // the rest of each head, and the values
  const int rest = (D - a.rot) / V, copied = H * rest, all = D / V;
  for (int i = tid; i < copied; i += kAppendT) {
    const int h = i / rest, d = a.rot + (i - h * rest) * V;
    if (T* out = to(h)) store(out + d, load(from(h) + d));
  }
  if (slot < 0) return;
  for (int i = tid; i < c.heads * all; i += kAppendT) {
    const int h = i / all, d = (i - h * all) * V;
    store(v_out + ((int64_t)h << log_ps) * D + d, load(v + (int64_t)h * D + d));
  }
  for (int h = tid; h < c.heads; h += kAppendT) {
    const int64_t at = ((int64_t)s * c.heads + h) * c.cap + slot;
    if (a.position) a.position[at] = pos;
    if (a.weight) a.weight[at] = 0.f;
  }
}

template <class T, int V>
static void launch_style(const AppendArgs& a, hipStream_t st) {
  if (a.interleaved)
    cache_append_rows<T, V, true><<<dim3(a.R), dim3(kAppendT), 0, st>>>(a);
  else
    cache_append_rows<T, V, false><<<dim3(a.R), dim3(kAppendT), 0, st>>>(a);
}

template <class T>
static hipError_t launch(const AppendArgs& a, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  auto whole = [](const void* p, int64_t stride) { return (uintptr_t)p % 16 == 0 && stride % V == 0; };
  if (a.rot % (2 * V) == 0 && whole(a.q, a.q_stride) && whole(a.k_new, a.k_stride) && whole(a.v_new, a.v_stride))
    launch_style<T, V>(a, st);
  else
    launch_style<T, 1>(a, st);
  return hipGetLastError();
}

hipError_t launch_cache_append(int bf16, const AppendArgs& a, hipStream_t st) {
  return bf16 ? launch<__bf16>(a, st) : launch<float>(a, st);
}

}  // namespace kb
