/*
 * kbest_loss.h -- C ABI of the output layer's losses: what trains the layer
 * that kbest.h decodes with, and what scores given translations under it.
 *
 * With logits x[n, j] = sum_i h[n, i] * W[i, j] + b[j] (h, W, b as for
 * kb_kbest_step: h N x H, W H x V, both row-major of one type, b float32):
 *
 *   kb_cross_entropy   loss[n] = lse[n] - (1 - s) x[n, t] - s / V sum_j x[n, j],
 *                      lse[n] = log sum_j exp(x[n, j]); t the row's target
 *                      word, s the label smoothing;
 *   kb_distill         with y = x / T, lse[n] = log sum_j exp(y[n, j]) and
 *                      q the softmax of the teacher's logits / T over the
 *                      words that it names for the row,
 *                      loss[n] = T^2 sum_j q_j (ln q_j - y[n, j] + lse[n]),
 *                      the T^2-fold divergence of the student's whole
 *                      distribution from q;
 *
 * and each one's gradient.  The N x V logits are never stored: the forward
 * pass keeps Algorithm 4's running (max, sum) of every row and the logits of
 * the words that count for it, the gradient works them out again from lse and
 * goes through the vocabulary in pieces, each of which is turned into its part
 * of all three gradients before the next.
 *
 * A row whose target is outside 0 .. V - 1 (padding), or none of whose
 * teacher's entries counts, is left out: its loss and lse are 0, it has no
 * part in any gradient, its row of dh is zeros, and its states are not read
 * (they may be anything).  Rows left out cost next to nothing.
 *
 * Conventions are those of kbest.h: device memory of the caller's, nothing
 * allocated, no synchronisation, work on `stream`, a kb_status back, nothing
 * enqueued on an error.  Calls on different streams are independent, given
 * different workspaces.  All calls may be captured into a HIP graph.  Results
 * do not depend on the order in which workgroups run: the same call gives the
 * same bits.  The states and logits of rows that count, W and the weights of
 * entries must be finite; b may be -inf for words that are to be left out
 * (not all of them).  The loss of a row whose target or whose smoothed labels
 * name such a word, or whose teacher gives one a probability above 0, is
 * +inf; its gradient is as it would be without that.  The gradient works from
 * x / T - lse in float32, so probabilities are as exact as a float32 lse of
 * that size is (2^-24 |lse|).
 *
 * Limits (KB_ERR_UNSUPPORTED beyond them): V <= KB_LOSS_MAX_V,
 * H <= KB_LOSS_MAX_H, N <= KB_LOSS_MAX_N, N * K <= 2^30.
 */
#ifndef KBEST_LOSS_H
#define KBEST_LOSS_H

#include "kbest.h"

#ifdef __cplusplus
extern "C" {
#endif

#define KB_LOSS_MAX_V 262144
#define KB_LOSS_MAX_H 65536
#define KB_LOSS_MAX_N 4194304
#define KB_LOSS_MAX_K 128 /* a teacher's entries of a row */

/*
 * Workspace bytes of kb_cross_entropy (K = 1) and kb_distill, and of their
 * gradients, whichever of the three are asked for.  0 for N = 0 and for sizes
 * that the calls refuse.  Never less for more rows, other sizes equal: a
 * workspace for the most rows that a program has at once serves all its
 * batches.
 * They grow with N * H (the states in bf16 pieces; gradients: dh in float32),
 * with N * K, and by N * V / 512 bytes (where the lists of the rows' words
 * begin); the gradients' by up to N * V / 8 besides (db's sums: a row for every
 * 32 rows, in large batches, N * V / 32, for every 128).  With the logits'
 * N * V and with H * V only as far as a piece of the vocabulary goes: of either
 * at most 256 MiB, or 256 words.
 */
size_t kb_loss_workspace_bytes(int dtype, int N, int H, int V, int K);
size_t kb_loss_grad_workspace_bytes(int dtype, int N, int H, int V, int K);

/*
 * kb_cross_entropy -- loss and log-sum-exp of every row.
 *   h, W, b       as for kb_kbest_step, aligned to their element size.
 *   target        N int32; outside 0 .. V - 1: the row is left out.
 *   smoothing     0 <= s < 1: the part of the labels spread over all words.
 *   loss, lse     N float32.
 *   workspace     kb_loss_workspace_bytes(dtype, N, H, V, 1) bytes,
 *                 256-byte aligned.
 * N = 0 is a no-op.
 */
kb_status kb_cross_entropy(int dtype, int N, int H, int V, const void* h, const void* W, const float* b,
                           const int32_t* target, float smoothing, float* loss, float* lse, void* workspace,
                           size_t workspace_bytes, void* stream);

/*
 * kb_cross_entropy_grad -- gradients of sum_n grad[n] * loss[n].
 *   lse           N float32, as kb_cross_entropy left it for the same h, W, b.
 *   grad          N float32 (those of rows left out are not read).
 *   dh            nullable, N x H of the type of h.
 *   dW            nullable, H x V of the type of W.
 *   db            nullable, V float32.
 * Outputs are overwritten, not added to, and may not overlap the inputs.  The
 * products take the logits' gradients rounded once: in bf16 to 2^-8, a
 * rounding as large as the results' own, for N <= 128 to 2^-17; in float32 to
 * 2^-24.  db is summed from them in float32 before that.  N = 0 gives zeros in
 * dW and db.
 *   workspace     kb_loss_grad_workspace_bytes(dtype, N, H, V, 1) bytes,
 *                 256-byte aligned.
 */
kb_status kb_cross_entropy_grad(int dtype, int N, int H, int V, const void* h, const void* W, const float* b,
                                const int32_t* target, float smoothing, const float* lse, const float* grad,
                                void* dh, void* dW, float* db, void* workspace, size_t workspace_bytes,
                                void* stream);

/*
 * kb_distill -- loss and log-sum-exp (of the logits / T) of every row against
 * a teacher's best words.
 *   K             entries of a row, 1 <= K <= KB_LOSS_MAX_K.
 *   token, logit  N x K int32 and float32, row-major, in any order: the
 *                 teacher's words and their logits (log-probabilities serve
 *                 as well: a row's constant drops out).  An entry whose token
 *                 is outside 0 .. V - 1 or whose logit / T is -inf counts for
 *                 nothing; entries of a row with the same token add up.
 *   temperature   1e-6 <= T <= 1e6; the logits / T must be finite.  The loss is
 *                 T^2 times sums of float32: off by a few 2^-24 T^2 |lse|.
 * The rest as for kb_cross_entropy; the workspace of K.
 */
kb_status kb_distill(int dtype, int N, int H, int V, int K, const void* h, const void* W, const float* b,
                     const int32_t* token, const float* logit, float temperature, float* loss, float* lse,
                     void* workspace, size_t workspace_bytes, void* stream);

/* kb_distill_grad -- gradients of sum_n grad[n] * loss[n]; lse from kb_distill.  The rest as for
 * kb_cross_entropy_grad. */
kb_status kb_distill_grad(int dtype, int N, int H, int V, int K, const void* h, const void* W, const float* b,
                          const int32_t* token, const float* logit, float temperature, const float* lse,
                          const float* grad, void* dh, void* dW, float* db, void* workspace,
                          size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KBEST_LOSS_H */
