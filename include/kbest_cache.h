/*
 * kbest_cache.h -- the attention cache of a decoder whose hypotheses attend
 * to their own past: keys and values in pages, the attention of one new token
 * a row over them, and their compaction to a budget.
 *
 * The output layer of kbest.h removes finished hypotheses from the batch
 * (kb_compact_*) and moves the per-hypothesis state of the others
 * (kb_gather_rows).  With attention that state is a page table: moving a
 * hypothesis moves its row of the table, the keys and values stay where they
 * are, and hypotheses of one sentence share the pages of their common past
 * (with pages of one slot, all of it).  Conventions (caller-owned device
 * buffers, stream ordering, kb_status returns, kb_last_error) are those of
 * kbest.h; the functions live in the same library.  In addition:
 *
 *  - Slot t of sequence s lies in page table[s * max_pages + t / page_size],
 *    place t % page_size.  A page outside [0, pages) is a hole: its slots are
 *    neither read, attended to nor written (kb_cache_evict counts them as
 *    slots all the same, see there).  Where slots are read, lengths above the
 *    table's max_pages * page_size are cut to that; negative ones are 0.  So
 *    no content of table, seq and length makes a call leave its buffers.
 *  - A call of R rows takes their count from the device where n_dev is given:
 *    min(R, *n_dev) rows are worked on, outputs of the others are left as
 *    they were.
 *  - Keys and values that no slot of a row's length refers to may hold
 *    anything, NaN and infinities included.
 *  - Results do not depend on the order in which workgroups run: no
 *    floating-point atomics.  The same call gives the same bits; in
 *    kb_cache_attend a row's last bits may differ with the lengths of the
 *    other rows, which move the places where its sums are cut and joined.
 */
#ifndef KBEST_CACHE_H
#define KBEST_CACHE_H

#include <stddef.h>
#include <stdint.h>

#include "kbest.h"

#ifdef __cplusplus
extern "C" {
#endif

#define KB_CACHE_MAX_DIM 256       /* largest head size                      */
#define KB_CACHE_MAX_PAGE 1024     /* largest page_size                      */
#define KB_CACHE_MAX_SLOTS (1 << 24) /* largest max_pages * page_size        */
#define KB_CACHE_MAX_EVICT (1 << 19) /* the largest that kb_cache_evict takes */

/* A cache: filled by the caller, read on the host during a call only. */
typedef struct kb_cache {
  int32_t dtype;        /* KB_F32 or KB_BF16: keys, values, queries, outputs */
  int32_t heads;        /* key-value heads, >= 1                             */
  int32_t dim;          /* head size: a multiple of 8, 8 .. KB_CACHE_MAX_DIM */
  int32_t page_size;    /* slots per page: a power of two, 1 .. 1024         */
  int32_t pages;        /* pages in k and in v                               */
  int32_t seqs;         /* rows of table                                     */
  int32_t max_pages;    /* columns of table                                  */
  void* k;              /* pages x heads x page_size x dim, 16-byte aligned  */
  void* v;              /* the same                                          */
  const int32_t* table; /* seqs x max_pages                                  */
} kb_cache;

/*
 * kb_cache_append -- the keys and values of R new tokens into their slots,
 * with rotary positions on queries and keys.
 *
 * Row r is a token of sequence s = seq[r] (r itself where seq is NULL; a
 * value outside [0, seqs) makes the row one of length 0) and goes to slot
 * length[r] - 1; a row whose length is below 1, or longer than the table has
 * slots, is not stored.  A prompt's tokens are rows with one seq and lengths
 * 1, 2, ...; where two rows of a call name the same place of a page, what it
 * holds afterwards is unspecified.  With m the amplitude and a_i = pos[r] *
 * freq[i], taken in 64 bits, each pair (x, y) of a query's or key's first
 * rot_dim values becomes
 *     (m (x cos a_i - y sin a_i), m (x sin a_i + y cos a_i)),   i < rot_dim / 2
 * rounded once; pair i is values (i, i + rot_dim / 2), or (2i, 2i + 1) where
 * interleaved.  The rest of the head, and values, are copied.  Positions
 * scaled for contexts longer than the trained ones are a matter of freq and
 * amplitude.
 *
 *   q_heads     heads of q; 0 where the call only stores (q and q_out NULL).
 *   q, k, v     rows of q_heads (k, v: cache heads) x dim values, one row
 *               q_stride (k_stride, v_stride) values after the other, so that
 *               the three may be parts of one fused projection's rows.  Any
 *               alignment to the element; 16-byte aligned rows are read in
 *               wide loads.  Not overlapping the cache or an output (q_out
 *               may be q where q_stride == q_heads * dim).
 *   rot_dim     even, 0 .. dim; 0: no rotation (pos, freq may be NULL).
 *   pos         R int32: rotary position of each row's token.
 *   freq        rot_dim / 2 doubles, radians per position.
 *   length      R int32.
 *   q_out       R x q_heads x dim: every row's rotated query (those of rows
 *               that are not stored too), 16-byte aligned.
 *   position    nullable; seqs x heads x (max_pages * page_size) int32:
 *               position[s, head, slot] = pos[r] (the slot where pos is
 *               NULL), for kb_cache_evict.
 *   weight      nullable; the same shape, float32: the new slot's is set to 0.
 * Errors: KB_ERR_INVALID_ARG for sizes out of range, null or misaligned
 * pointers; KB_ERR_UNSUPPORTED for sizes beyond the limits of kb_cache.
 */
kb_status kb_cache_append(const kb_cache* cache, int R, const int32_t* n_dev, int q_heads, const void* q,
                          int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                          int rot_dim, int interleaved, const int32_t* pos, const double* freq, float amplitude,
                          const int32_t* seq, const int32_t* length, void* q_out, int32_t* position, float* weight,
                          void* stream);

/*
 * kb_cache_attend -- attention of one new token a row over its cached slots:
 *     out[r, h] = sum_t p_t v[t],  p = softmax over t of scale * (q[r, h] . k[t])
 * t over the slots of [0, length[r]) that have a page, k and v of key-value
 * head h / (q_heads / heads).  A row with no such slot gets zeros and lse
 * -inf.  Scores, softmax and sums are float32; probabilities enter the second
 * product with at least 16 significand bits.  NaN or infinite queries, keys
 * or values of attended slots, and scores of 2e38 and more in magnitude, give
 * unspecified values in that row.
 *
 *   q_heads      a multiple of the cache's heads.
 *   q            rows of q_heads x dim values, q_stride values apart, aligned
 *                to the element.
 *   scale        finite, below 2e38 in magnitude.
 *   seq          nullable, R int32: table row of each row (r itself where
 *                NULL); rows may share one, as drafted tokens with lengths of
 *                their own do.
 *   length       R int32: slots to attend to, the new token's included.
 *   max_len      host-side bound of the lengths: longer ones are cut to it.
 *                At least 1; the work is split for it.
 *   out          R x q_heads x dim, 16-byte aligned; overlaps neither q nor the
 *                cache.
 *   lse          nullable, R x q_heads float32: log sum_t exp(score).
 *   weight_out   nullable, seqs x heads x (max_pages * page_size) float32:
 *                weight_out[r, head, t] = weight_in[r, head, t] + the sum of
 *                p_t over the query heads that share `head`, for every
 *                attended slot t; others are left as they were.  weight_in
 *                NULL counts as zeros; it may be weight_out.  Needs seq NULL
 *                (KB_ERR_UNSUPPORTED otherwise) and R <= seqs.
 *   workspace    kb_cache_attend_workspace_bytes(...) bytes, 256-byte
 *                aligned scratch (NULL allowed where that is 0); weights:
 *                nonzero where weight_out is given.  The bytes never shrink
 *                with R or max_len, so those of the largest call serve all.
 *                With weights they are at least 4 R q_heads max_len: give
 *                max_len where the table has far more slots than are used.
 */
size_t kb_cache_attend_workspace_bytes(const kb_cache* cache, int R, int q_heads, int max_len, int weights);
kb_status kb_cache_attend(const kb_cache* cache, int R, const int32_t* n_dev, int q_heads, const void* q,
                          int64_t q_stride, float scale, const int32_t* seq, const int32_t* length, int max_len,
                          void* out, float* lse, const float* weight_in, float* weight_out, void* workspace,
                          size_t workspace_bytes, void* stream);

/*
 * kb_cache_evict -- compaction of sequences that are over their budget: each
 * of the first R sequences keeps, head by head, the n = min(length, keep)
 * slots of greatest weight (kb_cache_attend's sums); equal weights keep the
 * lower slot, a NaN ranks below every number.  Slots whose position is below
 * `first` or above newest[r] - recent rank above all others, equal among
 * themselves.
 *
 * Kept slots below n stay where they are; the kept slots from n on fill, in
 * ascending order, the places of the dropped ones, so that as few keys and
 * values as possible move.  The order of a sequence's slots is then no longer
 * that of its tokens, which attention does not depend on; `position` keeps
 * it.  Rows are moved by the bits.
 *
 * Every slot below length, and every place below n of out_table, is to have a
 * page: attention over the n places is then attention over the kept slots.
 * Slots are ranked and placed by weight and position alone, and holes are not
 * looked for.  A kept slot that is a hole takes its weight and position to its
 * place, which goes on holding the key and value that lay there, to be
 * attended to if it has a page; a kept row whose place is a hole is lost.  A
 * sequence that has given pages up is therefore closed up first: its table's
 * remaining pages moved to the front, with the rows of weight and position
 * that go with them, and length cut to their slots.
 *
 *   length       R int32.
 *   keep         slots to keep, >= 1; first, recent >= 0, first + recent <=
 *                keep.
 *   newest       R int32: position of each sequence's newest token; may be
 *                NULL where recent is 0.
 *   weight       seqs x heads x (max_pages * page_size) float32.
 *   position     the same shape, int32; may be NULL where first and recent
 *                are 0.
 *   out_table    R x out_max_pages int32: the pages to keep the slots in,
 *                either the cache's own table (in place: out_table == table,
 *                out_max_pages == max_pages) or pages that hold none of the
 *                sequences' slots.  Sequences do not share these pages.
 *                out_max_pages * page_size >= min(keep, max_pages *
 *                page_size).
 *   out_length   R int32: n (may be length).
 *   out_weight   R x heads x (out_max_pages * page_size) float32: the kept
 *                slots' weights (may be weight where out_max_pages ==
 *                max_pages); places from n on are left as they were.
 *   out_position the same for position; NULL where position is.
 *   source       R x heads x keep int32: the slot that each kept place's row
 *                came from, -1 from n on.
 * Caches of more than KB_CACHE_MAX_EVICT slots a sequence: KB_ERR_UNSUPPORTED.
 */
kb_status kb_cache_evict(const kb_cache* cache, int R, const int32_t* n_dev, const int32_t* length, int keep, int first,
                         int recent, const int32_t* newest, const float* weight, const int32_t* position,
                         const int32_t* out_table, int out_max_pages, int32_t* out_length, float* out_weight,
                         int32_t* out_position, int32_t* source, void* stream);

#ifdef __cplusplus
} /* extern "C" */
#endif

#endif /* KBEST_CACHE_H */
