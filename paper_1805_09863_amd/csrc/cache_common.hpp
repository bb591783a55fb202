// The attention cache on the device: argument blocks and launchers of its
// three operators, and what their kernels share.
#pragma once

#include "kb_common.hpp"

namespace kb {

constexpr int kCacheMaxDim = 256;     // largest head size
constexpr int kEvictMax = 1 << 19;    // most slots of a sequence that eviction takes: their masks fit LDS

// A kb_cache as the kernels take it.
struct CacheView {
  void* k;               // pages x heads x page_size x dim
  void* v;
  const int32_t* table;  // seqs x max_pages
  int heads, dim, log_ps, pages, seqs, max_pages, cap;  // cap = max_pages << log_ps
};

struct AppendArgs {
  CacheView c;
  int R, q_heads, rot, interleaved;
  const int32_t* n_dev;
  const void *q, *k_new, *v_new;
  int64_t q_stride, k_stride, v_stride;
  const int32_t* pos;
  const double* freq;
  float amplitude;
  const int32_t* seq;
  const int32_t* length;
  void* q_out;
  int32_t* position;
  float* weight;
};

struct AttendArgs {
  CacheView c;
  int R, q_heads, max_len;
  const int32_t* n_dev;
  const void* q;
  int64_t q_stride;
  float scale;
  const int32_t* seq;
  const int32_t* length;
  void* out;
  float* lse;
  const float* weight_in;
  float* weight_out;
  // the launch: waves per workgroup, tiles of 16 query heads per key-value head, splits of `chunk` slots; or
  // (shared) equal shares of all rows' slots
  int waves, head_tiles, chunk, splits, shared;
  // workspace: partial outputs (dim floats) and their (max, sum), in base 2: one per row, query head and
  // split (splits > 1), or 16 query heads' two per share, and the costs before each row; with weight_out the
  // scores in base 2, score_ld apart per row and query head, and the (max, 1 / sum) of those that the pass
  // finishes
  float* part_o;
  float2* part_s;
  int* row_before;
  float* scores;
  float2* finished;
  int64_t score_ld;
  int weight_blocks;  // of the second launch, a (row, key-value head); the others join
};

// Attention's slots in equal shares, where lengths differ or splits would start and end too often.
// Every (key-value head, 16 query heads), one after the other, has all rows in order; a row costs its
// steps (the slots that a workgroup takes at a time) and kStart more for starting on it (a call of 64 x 8 of up
// to 8,192 slots: 59 us at 1, 56 at 2, 60 at 4; with weights 82, 83 and 87).
// Share b is the b-th of kShares equal parts of all of it, one workgroup's: a row within one share is
// finished there, one that shares cut leaves a partial in each, which the join adds up.  A share cuts at
// most two: the one it starts within and the one it ends within.
constexpr int kShareRows = 1024;
constexpr int kShares = 256;  // workgroups; a power of two and a multiple of the 8 XCDs
struct AttendShares {
  long long total;
  int shares;  // no more than total: none is empty
  // all: the cost of all rows, for one (key-value head, 16 query heads); columns: how many of these there are
  __device__ __forceinline__ AttendShares(int all, int columns)
      : total((long long)all * columns), shares((int)min((long long)kShares, total)) {}
  static constexpr int kStart = 1;
  static __device__ __forceinline__ int cost(int len, int step) { return (len + step - 1) / step + kStart; }
  // The first slot of a row at place o of its cost; the start's places come first.
  static __device__ __forceinline__ int slot(int o, int step) { return max(o - kStart, 0) * step; }
  __device__ __forceinline__ long long begin(int b) const { return shares < kShares ? b : b * total / kShares; }
  // The share that x lies in: the largest b with begin(b) <= x.
  __device__ __forceinline__ int of(long long x) const {
    if (shares < kShares) return (int)x;
    const long long n = (x + 1) * kShares - 1;
    return total <= UINT_MAX / kShares ? (int)((uint32_t)n / (uint32_t)total) : (int)(n / total);
  }
  static __device__ __forceinline__ int64_t partial(int b, int o0) { return 2 * (int64_t)b + (o0 == 0 ? 1 : 0); }
};

struct EvictArgs {
  CacheView c;
  int R, keep, first, recent, out_max_pages;
  const int32_t* n_dev;
  const int32_t* length;
  const int32_t* newest;
  const float* weight;
  const int32_t* position;
  const int32_t* out_table;
  int32_t* out_length;
  float* out_weight;
  int32_t* out_position;
  int32_t* source;
  int units;  // 16-byte pieces of a row
};

hipError_t launch_cache_append(int bf16, const AppendArgs& a, hipStream_t st);
hipError_t launch_cache_attend(int bf16, AttendArgs& a, hipStream_t st);
hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t st);

// Row (of dim values, in k or v) of slot t of a sequence whose table row is
// `pages`, for key-value head `head`; -1 for a hole.  Rows are counted in 32
// bits (the host refuses pools of 2^31 and more), their bytes in 64.
__device__ __forceinline__ int cache_row(const CacheView& c, const int32_t* pages, int head, int t) {
  const int page = pages[t >> c.log_ps];
  if ((uint32_t)page >= (uint32_t)c.pages) return -1;
  return ((page * c.heads + head) << c.log_ps) + (t & ((1 << c.log_ps) - 1));
}

// Table row of row r of a call, -1 where seq names none.
__device__ __forceinline__ int cache_seq(const CacheView& c, const int32_t* seq, int r) {
  const int s = seq ? seq[r] : r;
  return (uint32_t)s < (uint32_t)c.seqs ? s : -1;
}

__device__ __forceinline__ int rows_of(int R, const int32_t* n_dev) { return n_dev ? max(0, min(R, *n_dev)) : R; }

}  // namespace kb
