/*
 * pbg_operators.h -- operators on a caller's own tensors, beside the bucket-training calls of pbg.h and in the
 * same library: what a training step other than the built-in one is made of.
 *
 *   pbg_group_linear / _backward      products with one matrix per group of rows: the LINEAR operator for rows grouped
 *                                     by relation (or by expert), with both gradients
 *   pbg_preference_loss / _backward   loss on preferred and other sequences of candidate scores (paired log ratios)
 *   pbg_clip_gradients                the joint norm of many gradients, and their scaling to a bound
 *
 * Conventions are those of pbg.h: a pbg_status from every call, a message in pbg_last_error, device pointers unless a
 * name ends in _host, work on the context's compute stream (pbg_set_streams), every call synchronous on return, nothing
 * written on an error (a HIP failure while the work runs excepted), the same inputs give the same bits.  The context
 * supplies device, stream and workspace; its graph (entities, relations, operator) does not matter here, and contexts
 * with entity types serve too.  The context's device must be current (else STATE).  Because the calls wait for
 * their work they cannot be recorded into a HIP graph: on a capturing stream they return STATE and leave the capture
 * as it is.
 *
 * Matrices of rows take a row stride (ld, in elements) of at least their width and at most PBG_OPS_MAX_LD; columns are
 * consecutive.  Element pointers must be aligned to their element, nothing more; rows that start at multiples of 16
 * bytes are read fastest (the grouped products first copy operands whose rows do not into the workspace, which grows to
 * hold them: of the groups' matrices only those of groups that have rows, and no more than there are rows).  Arrays
 * lie on the context's device.  An output may not overlap an input or another output unless stated (INVALID_ARG; two
 * matrices with the same row stride and type may share rows' memory in columns of their own).
 */
#ifndef PBG_OPERATORS_H
#define PBG_OPERATORS_H

#include "pbg.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  Sums are formed in float32 or wider whatever the type; results are rounded to the type once (to
 * nearest, ties to even). */
enum { PBG_TYPE_F32 = 0, PBG_TYPE_BF16 = 1, PBG_TYPE_F16 = 2 };

#define PBG_OPS_MAX_LD (1 << 20)     /* largest row stride, in elements */
#define PBG_OPS_MAX_DIM (1 << 16)    /* largest in_dim, out_dim */
#define PBG_OPS_MAX_GROUPS (1 << 20) /* largest number of groups or sequences */

/* y[t, :] = A_g x[t, :] for the rows t in [offsets[g], offsets[g+1]) of group g (Sec. 3.1 operator table, g(x) = A_r x,
 * A_g row-major [out_dim x in_dim], for edges grouped by relation as pbg_group_by_relation leaves them; also a layer of
 * experts over tokens grouped by expert, or with one group a plain product x A^T, e.g. candidate scores).
 * x [n x in_dim] (row stride ldx), a [groups x out_dim x in_dim] contiguous and y [n x out_dim] (row stride ldy) share
 * the type dtype; offsets [groups + 1] int64 (device), nondecreasing, within [0, n].  Groups may be empty; rows of y
 * outside [offsets[0], offsets[groups]) are left as they are.  n <= 2^31 - 1; arrays may be NULL when n is 0.
 * INVALID_ARG for offsets that decrease or leave [0, n]. */
pbg_status pbg_group_linear(pbg_ctx* ctx, int32_t dtype, const void* x, int64_t ldx, const void* a,
                            const int64_t* offsets, int32_t groups, int64_t n, int32_t in_dim, int32_t out_dim,
                            void* y, int64_t ldy);

/* Gradients of pbg_group_linear for dy [n x out_dim] (row stride lddy):
 *   dx[t, :] = A_g^T dy[t, :]                 [n x in_dim], row stride lddx; rows outside every group left as they are
 *   da_g = sum over g's rows of dy[t, :] x[t, :]^T   [groups x out_dim x in_dim] contiguous; zeros for an empty group
 * Either output may be NULL (not wanted); then x (needed for da only) or a (needed for dx only) may be NULL too. */
pbg_status pbg_group_linear_backward(pbg_ctx* ctx, int32_t dtype, const void* x, int64_t ldx, const void* a,
                                     const void* dy, int64_t lddy, const int64_t* offsets, int32_t groups, int64_t n,
                                     int32_t in_dim, int32_t out_dim, void* dx, int64_t lddx, void* da);

/* Loss on pairs of sequences (a preferred path of edges against another one; Sec. 3.1 SOFTMAX gives each row's
 * log probability).  Rows [offsets[q], offsets[q+1]) of logits [n x candidates] (row stride ld, type dtype) belong to
 * sequence q of 2 pairs sequences; sequence 2p is preferred over 2p + 1.  labels [n] int32 holds each row's candidate,
 * negative where the row does not count.  A candidate is left out of a row's distribution by a score of -inf; a row
 * whose scores are all -inf does not count either.  With l_t = logits[t, y_t] - log sum_v exp(logits[t, v]):
 *   logp[q]   = sum of l_t over q's rows that count (0 if there are none)
 *   h_p       = beta ((logp[2p] - ref[2p]) - (logp[2p+1] - ref[2p+1]))
 *   loss[p]   = (1 - smoothing) softplus(-h_p) + smoothing softplus(h_p)
 *   dlogp[q]  = d loss[p] / d logp[q]
 *   row_stats[t] = (largest score m of row t, log sum_v exp(logits[t, v] - m)); (0, 0) where y_t < 0, (-inf, 0) where
 *               every score is -inf; left as it is for rows outside every sequence
 * ref_logp [2 pairs] float32 (the frozen model's logp; NULL: zeros); loss [pairs], logp, dlogp [2 pairs] and
 * row_stats [n x 2] are float32; loss and dlogp may be NULL (a frozen model's pass).  A score of NaN or +inf in a row
 * that counts makes the row's log sum NaN (sums go over exp(logits[t, v] - m), and inf - inf is no number), and with it
 * l_t, logp[q] and its pair's loss, dlogp and gradients; a label that is left out gives l_t = -inf.  offsets [2 pairs + 1]
 * int64 as in pbg_group_linear; beta finite, smoothing in [0, 1); candidates <= PBG_OPS_MAX_LD; pairs in
 * [1, PBG_OPS_MAX_GROUPS / 2]; n < 2^24.  INVALID_ARG for bad offsets and for a label of a row inside a sequence that is
 * >= candidates. */
pbg_status pbg_preference_loss(pbg_ctx* ctx, int32_t dtype, const void* logits, int64_t ld, const int32_t* labels,
                               const int64_t* offsets, int32_t pairs, int64_t n, int32_t candidates,
                               const float* ref_logp, float beta, float smoothing, float* loss, float* logp,
                               float* dlogp, float* row_stats);

/* dlogits[t, v] = dlogp[q] ([v = y_t] - exp(logits[t, v] - m_t - s_t)) for the rows that count of every sequence q, with
 * (m_t, s_t) = row_stats[t] as pbg_preference_loss left them and dlogp as it left them or as the caller scaled them
 * (d total loss / d logp[q]); zeros for rows of a sequence that do not count; rows outside every sequence are left as
 * they are.  dlogits [n x candidates] has the type of logits and row stride lddl, and may be logits itself
 * (the same pointer and stride). */
pbg_status pbg_preference_loss_backward(pbg_ctx* ctx, int32_t dtype, const void* logits, int64_t ld,
                                        const int32_t* labels, const int64_t* offsets, int32_t pairs, int64_t n,
                                        int32_t candidates, const float* row_stats, const float* dlogp, void* dlogits,
                                        int64_t lddl);

/* The joint norm of num_tensors gradients, sqrt(sum of all squares), and their scaling to at most max_norm:
 *   outs[i] = grads[i] * min(1, max_norm / norm)
 * dtypes_host [num_tensors] int32 (PBG_TYPE_*), counts_host [num_tensors] int64 (elements, at most 2^38 together; 0
 * is allowed, with NULL pointers),
 * grads_host and outs_host [num_tensors] host arrays of device pointers to contiguous values.  outs_host NULL, or
 * outs_host[i] equal to grads_host[i]: in place.  No output may overlap another tensor (INVALID_ARG).  max_norm > 0;
 * +inf: only the norm (in place nothing is written).  norm_host (nullable) receives the norm.  Squares are summed in
 * float64, so the norm neither overflows nor loses small gradients; a norm that is not finite scales nothing (outputs
 * that are not in place receive copies). */
pbg_status pbg_clip_gradients(pbg_ctx* ctx, int32_t num_tensors, const int32_t* dtypes_host, const int64_t* counts_host,
                              const void* const* grads_host, void* const* outs_host, double max_norm,
                              double* norm_host);

#ifdef __cplusplus
}
#endif

#endif /* PBG_OPERATORS_H */
