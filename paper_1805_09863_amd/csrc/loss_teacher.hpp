// A teacher's row: the softmax over its entries' words of logit / T, by one wave, up to two entries a lane (entry
// lane + 64 u).  An entry whose word is outside the vocabulary or whose logit is -inf is none; entries of the same word
// are one, the first, with their probabilities' sum.
#pragma once

#include "loss_common.hpp"

namespace kb {

struct TeacherRow {
  int token[2];   // -1: no entry, or an earlier one has the same word
  float part[2];  // the word's probability
  float known;    // sum q ln q
  bool any;
};

__device__ __forceinline__ TeacherRow teacher_row(const int32_t* token, const float* logit, int K, int V, float inv_t) {
  const int lane = threadIdx.x & 63;
  int tok[2];
  float y[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int j = lane + 64 * u;
    tok[u] = -1;
    y[u] = -INFINITY;
    if (j < K) {
      const int t = token[j];
      const float x = logit[j] * inv_t;
      if (t >= 0 && t < V && !(x == -INFINITY)) {
        tok[u] = t;
        y[u] = x;
      }
    }
  }
  TeacherRow r;
  r.any = __builtin_amdgcn_ballot_w64(tok[0] >= 0 || tok[1] >= 0) != 0ull;
  float top = fmaxf(y[0], y[1]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  float e[2], merged[2], total = 0.f;
  bool first[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    e[u] = tok[u] >= 0 ? expf(y[u] - top) : 0.f;
    merged[u] = 0.f;
    total += e[u];
    first[u] = tok[u] >= 0;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d, 64);
#pragma unroll
  for (int u = 0; u < 2; ++u)
    for (int i = 0; i < min(64, K - 64 * u); ++i) {
      const int t = __builtin_amdgcn_readlane(tok[u], i);
      const float x = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e[u]), i));
      const auto same = [&](int w) {
        if (t >= 0 && t == tok[w]) {
          merged[w] += x;
          if (i + 64 * u < lane + 64 * w) first[w] = false;
        }
      };
      same(0);
      if (K > 64) same(1);
    }
  r.known = 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const float q = first[u] ? merged[u] / total : 0.f;
    if (q > 0.f) r.known += q * (logf(merged[u]) - logf(total));
    if (first[u] && !(q >= 0.f)) r.known = q;  // NaN stays NaN
    r.token[u] = first[u] ? tok[u] : -1;
    r.part[u] = q;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) r.known += __shfl_xor(r.known, d, 64);
  return r;
}

}  // namespace kb
