// Host side of the attention cache: argument validation and the entry points
// declared in include/kbest_cache.h.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "cache_common.hpp"
#include "kb_status.hpp"
#include "kbest_cache.h"

namespace {

using kb::aligned;
using kb::fail;
using kb::ok;

static_assert(kb::kCacheMaxDim == KB_CACHE_MAX_DIM && kb::kEvictMax == KB_CACHE_MAX_EVICT, "the same limits");

kb_status check_cache(const kb_cache* c) {
  if (!c) return fail(KB_ERR_INVALID_ARG, "null cache");
  if (c->dtype != KB_F32 && c->dtype != KB_BF16) return fail(KB_ERR_INVALID_ARG, "unknown dtype %d", c->dtype);
  if (c->heads < 1) return fail(KB_ERR_INVALID_ARG, "heads = %d must be >= 1", c->heads);
  if (c->dim < 8 || c->dim > KB_CACHE_MAX_DIM || c->dim % 8 != 0)
    return fail(KB_ERR_INVALID_ARG, "dim = %d: a multiple of 8 up to %d", c->dim, KB_CACHE_MAX_DIM);
  if (c->page_size < 1 || c->page_size > KB_CACHE_MAX_PAGE || (c->page_size & (c->page_size - 1)) != 0)
    return fail(KB_ERR_INVALID_ARG, "page_size = %d: a power of two up to %d", c->page_size, KB_CACHE_MAX_PAGE);
  if (c->pages < 0 || c->seqs < 0 || c->max_pages < 1)
    return fail(KB_ERR_INVALID_ARG, "pages = %d, seqs = %d, max_pages = %d", c->pages, c->seqs, c->max_pages);
  if ((long long)c->max_pages * c->page_size > KB_CACHE_MAX_SLOTS)
    return fail(KB_ERR_UNSUPPORTED, "max_pages * page_size = %lld exceeds %d", (long long)c->max_pages * c->page_size,
                KB_CACHE_MAX_SLOTS);
  // in this order no product leaves 64 bits
  if ((long long)c->pages * c->page_size > INT_MAX || (long long)c->pages * c->page_size * c->heads > INT_MAX)
    return fail(KB_ERR_UNSUPPORTED, "pages * heads * page_size exceeds INT_MAX");
  if ((long long)c->seqs * c->heads > INT_MAX) return fail(KB_ERR_UNSUPPORTED, "seqs * heads exceeds INT_MAX");
  return KB_OK;
}

kb_status check_pointers(const kb_cache* c) {
  if ((c->pages > 0 && (!c->k || !c->v)) || (c->seqs > 0 && !c->table))
    return fail(KB_ERR_INVALID_ARG, "null k, v or table");
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return fail(KB_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  if (!aligned(c->table, 4)) return fail(KB_ERR_INVALID_ARG, "table must be 4-byte aligned");
  return KB_OK;
}

kb::CacheView view(const kb_cache* c) {
  return {c->k,     c->v,    c->table,     c->heads,                        c->dim, __builtin_ctz(c->page_size),
          c->pages, c->seqs, c->max_pages, c->max_pages * c->page_size};
}

// R rows of `heads` heads, `stride` values apart.
kb_status check_rows(const char* what, const kb_cache* c, const void* p, int64_t stride, int heads) {
  if (!p) return fail(KB_ERR_INVALID_ARG, "null %s", what);
  if (!aligned(p, c->dtype == KB_BF16 ? 2 : 4)) return fail(KB_ERR_INVALID_ARG, "%s not aligned to its type", what);
  if (stride < (int64_t)heads * c->dim || stride > ((int64_t)1 << 40))
    return fail(KB_ERR_INVALID_ARG, "%s rows %lld values apart hold no %d x %d", what, (long long)stride, heads,
                c->dim);
  return KB_OK;
}

kb_status check_count(int R, int q_heads) {
  if (R < 0) return fail(KB_ERR_INVALID_ARG, "R = %d < 0", R);
  if ((long long)R * std::max(q_heads, 1) > INT_MAX / KB_CACHE_MAX_DIM)
    return fail(KB_ERR_UNSUPPORTED, "R * heads = %lld too large", (long long)R * q_heads);
  return KB_OK;
}

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

struct AttendPlan {
  int waves, head_tiles, chunk, splits, shared;
  size_t score_ld, part_o, part_s, row_before, scores, finished, bytes;  // workspace offsets
};

AttendPlan attend_plan(const kb_cache* c, int R, int q_heads, int max_len, bool weights) {
  AttendPlan p{};
  max_len = std::min(max_len, c->max_pages * c->page_size);
  const int group = q_heads / c->heads;
  p.head_tiles = (group + 15) / 16;
  // (Times are whole calls on the device, replayed from a graph of ten over two caches in turn; bf16 heads of
  // 128 but where stated.)
  // A unit is a row's slots for 16 query heads.  Where units fill the card and are at most 64 slots long,
  // one wave takes each (640 rows x 8 heads of up to 60 slots: 14.2 us, four waves 27.5), else four take its
  // tiles in turn (5 x 16 of up to 60, float32 heads of 64: 5.1 us, one wave 6.8).
  const long long units = (long long)R * c->heads * p.head_tiles;
  p.waves = max_len <= 64 && units >= 1024 ? 1 : 4;
  // Beyond 6 steps of the four waves the slots are shared out: 256 workgroups take equal parts of all rows
  // (64 x 8 of up to 8,192: 59 us, splits of 1,024 slots 71; 128 x 8 of 4,096: 377, splits 395; one row of
  // 131,072: 103 and 104; 512 workgroups 58, 374 and 104).  Up to there, where the join's launch would cost
  // more than it gives (4 x 8 of 300: 7.6 us, shared out 10.9; 1 x 8 of 600: 9.8 and 10.4; in float32, whose steps
  // are half as long, 4 x 8 of 300: 12.7 and 12.2), each row is one workgroup's; and with more rows than the
  // shares' kernel can add up, splits of 1,024 slots are.
  const int step = c->dtype == KB_BF16 ? 128 : 64;
  const bool long_rows = max_len > 6 * step;
  p.shared = long_rows && R <= kb::kShareRows;
  p.chunk = p.shared ? max_len : std::min(max_len, R <= kb::kShareRows ? 6 * step : 1024);
  p.splits = (max_len + p.chunk - 1) / p.chunk;
  const size_t rh = (size_t)R * q_heads;
  // Never less for more rows or longer ones, so that a workspace for the largest call serves all: rows that
  // are one workgroup's because there are many of them still ask for what fewer would need for their shares.
  const size_t least = (size_t)kb::kShares * 2 * 16;
  const size_t parts = p.splits > 1 ? std::max(least, rh * p.splits) : long_rows ? least : 0;
  if (parts > 0) {
    p.part_s = align_up(parts * c->dim * sizeof(float), 256);
    p.row_before = align_up(p.part_s + parts * sizeof(float2), 256);
    p.bytes = align_up(p.row_before + ((size_t)R + 1) * sizeof(int), 256);
  }
  if (weights) {
    p.score_ld = align_up(max_len, 32);
    p.scores = p.bytes;
    p.finished = align_up(p.scores + rh * p.score_ld * sizeof(float), 256);
    p.bytes = align_up(p.finished + rh * sizeof(float2), 256);
  }
  return p;
}

bool bf16(const kb_cache* c) { return c->dtype == KB_BF16; }

}  // namespace

extern "C" {

kb_status kb_cache_append(const kb_cache* cache, int R, const int32_t* n_dev, int q_heads, const void* q,
                          int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                          int rot_dim, int interleaved, const int32_t* pos, const double* freq, float amplitude,
                          const int32_t* seq, const int32_t* length, void* q_out, int32_t* position, float* weight,
                          void* stream) {
  kb_status st = check_cache(cache);
  if (st != KB_OK) return st;
  if (q_heads < 0) return fail(KB_ERR_INVALID_ARG, "q_heads = %d < 0", q_heads);
  if ((st = check_count(R, std::max(q_heads, cache->heads))) != KB_OK) return st;
  if (rot_dim < 0 || rot_dim > cache->dim || rot_dim % 2 != 0)
    return fail(KB_ERR_INVALID_ARG, "rot_dim = %d: even, up to dim = %d", rot_dim, cache->dim);
  if (R == 0) return ok();
  if ((st = check_pointers(cache)) != KB_OK) return st;
  if (q_heads > 0) {
    if ((st = check_rows("q", cache, q, q_stride, q_heads)) != KB_OK) return st;
    if (!q_out || !aligned(q_out, 16)) return fail(KB_ERR_INVALID_ARG, "q_out null or not 16-byte aligned");
  } else if (q || q_out) {
    return fail(KB_ERR_INVALID_ARG, "q or q_out without q_heads");
  }
  if ((st = check_rows("k", cache, k, k_stride, cache->heads)) != KB_OK) return st;
  if ((st = check_rows("v", cache, v, v_stride, cache->heads)) != KB_OK) return st;
  if (!length) return fail(KB_ERR_INVALID_ARG, "null length");
  if (rot_dim > 0 && (!pos || !freq)) return fail(KB_ERR_INVALID_ARG, "rotation needs pos and freq");
  if (!aligned(freq, 8)) return fail(KB_ERR_INVALID_ARG, "freq not aligned to its type");
  if (!isfinite(amplitude)) return fail(KB_ERR_INVALID_ARG, "amplitude is not finite");
  if (!seq && R > cache->seqs) return fail(KB_ERR_INVALID_ARG, "R = %d rows, seqs = %d and no seq", R, cache->seqs);
  const kb::AppendArgs a{view(cache), R,    q_heads, rot_dim,   interleaved != 0, n_dev,  q,        k,     v,
                         q_stride,    k_stride, v_stride, pos, freq, amplitude, seq, length, q_out, position, weight};
  hipError_t e = kb::launch_cache_append(bf16(cache), a, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(KB_ERR_HIP, "cache append kernel launch: %s", hipGetErrorString(e));
  return ok();
}

size_t kb_cache_attend_workspace_bytes(const kb_cache* cache, int R, int q_heads, int max_len, int weights) {
  if (check_cache(cache) != KB_OK || q_heads < 1 || q_heads % cache->heads != 0 || max_len < 1 ||
      check_count(R, q_heads) != KB_OK || R == 0)
    return 0;
  return attend_plan(cache, R, q_heads, max_len, weights != 0).bytes;
}

kb_status kb_cache_attend(const kb_cache* cache, int R, const int32_t* n_dev, int q_heads, const void* q,
                          int64_t q_stride, float scale, const int32_t* seq, const int32_t* length, int max_len,
                          void* out, float* lse, const float* weight_in, float* weight_out, void* workspace,
                          size_t workspace_bytes, void* stream) {
  kb_status st = check_cache(cache);
  if (st != KB_OK) return st;
  if (q_heads < 1 || q_heads % cache->heads != 0)
    return fail(KB_ERR_INVALID_ARG, "q_heads = %d is no multiple of heads = %d", q_heads, cache->heads);
  if ((st = check_count(R, q_heads)) != KB_OK) return st;
  if (max_len < 1) return fail(KB_ERR_INVALID_ARG, "max_len = %d < 1", max_len);
  if (!isfinite(scale * kb::kL2E)) return fail(KB_ERR_INVALID_ARG, "scale is not finite, or too large");
  if (R == 0) return ok();
  if ((st = check_pointers(cache)) != KB_OK) return st;
  if ((st = check_rows("q", cache, q, q_stride, q_heads)) != KB_OK) return st;
  if (!length) return fail(KB_ERR_INVALID_ARG, "null length");
  if (!out || !aligned(out, 16)) return fail(KB_ERR_INVALID_ARG, "out null or not 16-byte aligned");
  if (!seq && R > cache->seqs) return fail(KB_ERR_INVALID_ARG, "R = %d rows, seqs = %d and no seq", R, cache->seqs);
  if (weight_in && !weight_out) return fail(KB_ERR_INVALID_ARG, "weight_in without weight_out");
  if (weight_out && seq) return fail(KB_ERR_UNSUPPORTED, "weights need a table row for each row (seq NULL)");
  const AttendPlan p = attend_plan(cache, R, q_heads, max_len, weight_out != nullptr);
  if ((long long)R * cache->heads * p.head_tiles * p.splits * p.waves * 64 > UINT32_MAX)  // threads of a launch
    return fail(KB_ERR_UNSUPPORTED, "R * heads * %d splits too large", p.splits);
  if (p.bytes > 0) {
    if (!workspace) return fail(KB_ERR_WORKSPACE, "workspace is null (%zu bytes needed)", p.bytes);
    if (!aligned(workspace, 256)) return fail(KB_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    if (workspace_bytes < p.bytes)
      return fail(KB_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", workspace_bytes, p.bytes);
  }
  char* ws = static_cast<char*>(workspace);
  kb::AttendArgs a{view(cache), R,      q_heads, max_len, n_dev, q,         q_stride,
                   scale,       seq, length,  out,     lse,   weight_in, weight_out};
  // no length counts where there is nothing to attend to
  a.max_len = cache->pages == 0 || cache->seqs == 0 ? 0 : std::min(max_len, cache->max_pages * cache->page_size);
  a.waves = p.waves;
  a.head_tiles = p.head_tiles;
  a.chunk = p.chunk;
  a.splits = p.splits;
  a.shared = a.max_len > 0 && p.shared;
  if (p.splits > 1 || p.shared) {
    a.part_o = reinterpret_cast<float*>(ws + p.part_o);
    a.part_s = reinterpret_cast<float2*>(ws + p.part_s);
    a.row_before = reinterpret_cast<int*>(ws + p.row_before);
  }
  if (weight_out) {
    a.scores = reinterpret_cast<float*>(ws + p.scores);
    a.score_ld = (int64_t)p.score_ld;
    a.finished = reinterpret_cast<float2*>(ws + p.finished);
  }
  hipError_t e = kb::launch_cache_attend(bf16(cache), a, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(KB_ERR_HIP, "cache attention kernel launch: %s", hipGetErrorString(e));
  return ok();
}

kb_status kb_cache_evict(const kb_cache* cache, int R, const int32_t* n_dev, const int32_t* length, int keep, int first,
                         int recent, const int32_t* newest, const float* weight, const int32_t* position,
                         const int32_t* out_table, int out_max_pages, int32_t* out_length, float* out_weight,
                         int32_t* out_position, int32_t* source, void* stream) {
  kb_status st = check_cache(cache);
  if (st != KB_OK) return st;
  if ((st = check_count(R, cache->heads)) != KB_OK) return st;
  if ((long long)R * cache->heads * 1024 > UINT32_MAX)  // threads of a launch
    return fail(KB_ERR_UNSUPPORTED, "R * heads = %lld too large", (long long)R * cache->heads);
  if (keep < 1 || first < 0 || recent < 0 || (long long)first + recent > keep)
    return fail(KB_ERR_INVALID_ARG, "keep = %d, first = %d, recent = %d", keep, first, recent);
  const int cap = cache->max_pages * cache->page_size;
  if (cap > KB_CACHE_MAX_EVICT)
    return fail(KB_ERR_UNSUPPORTED, "max_pages * page_size = %d exceeds %d", cap, KB_CACHE_MAX_EVICT);
  if (out_max_pages < 1 || (long long)out_max_pages * cache->page_size < std::min(keep, cap))
    return fail(KB_ERR_INVALID_ARG, "out_max_pages = %d of %d slots hold no %d", out_max_pages, cache->page_size,
                std::min(keep, cap));
  if (keep > KB_CACHE_MAX_SLOTS || (long long)out_max_pages * cache->page_size > KB_CACHE_MAX_SLOTS)
    return fail(KB_ERR_UNSUPPORTED, "keep or out_max_pages * page_size exceeds %d", KB_CACHE_MAX_SLOTS);
  if (R == 0) return ok();
  if ((st = check_pointers(cache)) != KB_OK) return st;
  if (R > cache->seqs) return fail(KB_ERR_INVALID_ARG, "R = %d exceeds seqs = %d", R, cache->seqs);
  if (!length || !weight || !out_table || !out_length || !out_weight || !source)
    return fail(KB_ERR_INVALID_ARG, "null length, weight, out_table, out_length, out_weight or source");
  if ((position == nullptr) != (out_position == nullptr))
    return fail(KB_ERR_INVALID_ARG, "position and out_position: both or neither");
  if ((first > 0 || recent > 0) && !position) return fail(KB_ERR_INVALID_ARG, "first and recent need position");
  if (recent > 0 && !newest) return fail(KB_ERR_INVALID_ARG, "recent needs newest");
  if (out_table == cache->table && out_max_pages != cache->max_pages)
    return fail(KB_ERR_INVALID_ARG, "in place, out_max_pages is max_pages = %d", cache->max_pages);
  if ((out_weight == weight || (position && out_position == position)) && out_max_pages != cache->max_pages)
    return fail(KB_ERR_INVALID_ARG, "out_weight and out_position of another row length cannot be weight and position");
  const kb::EvictArgs a{view(cache), R,      keep,     first,     recent,     out_max_pages, n_dev,        length,
                        newest,      weight, position, out_table, out_length, out_weight,    out_position, source,
                        cache->dim * (bf16(cache) ? 2 : 4) / 16};
  hipError_t e = kb::launch_cache_evict(a, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(KB_ERR_HIP, "cache eviction kernel launch: %s", hipGetErrorString(e));
  return ok();
}

}  // extern "C"
