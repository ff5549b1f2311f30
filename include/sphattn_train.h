/*
 * sphattn -- what a model that trains with the attention of sphattn.h has at its two ends, C ABI:
 * the lookup of gene-token embeddings, the cross entropy over the vocabulary, and the clipping of
 * gradients before the optimizer.
 *
 * Conventions are those of sphattn.h: device pointers owned by the caller, nothing allocated, no state,
 * work enqueued on `stream` without synchronising, one of sphattn.h's return codes.  dtype is
 * SPHATTN_F32, SPHATTN_BF16 or SPHATTN_F16 (SPHATTN_ERR_DTYPE otherwise).  All tensors are contiguous;
 * pointers need the alignment of one element only (rows that are whole multiples of 16 bytes from a
 * 16-byte-aligned start on are faster), workspaces 16 bytes.  Outputs overlap neither each other nor
 * inputs nor the workspace unless stated (SPHATTN_ERR_ALIAS).  Calls that share a workspace must be ordered.
 * Results do not depend on the order in which workgroups run: no float is added atomically.
 *
 * Token ids and targets are int32 (id_bytes 4) or int64 (id_bytes 8); other id_bytes return SPHATTN_ERR_DTYPE.
 * T == 0 is allowed everywhere (outputs of no rows; gradients of tables are zeros).
 */
#ifndef SPHATTN_TRAIN_H
#define SPHATTN_TRAIN_H

#include "sphattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Rows of a table, scaled:  O[t,:] = scale * mult[t] * table[tokens[t],:]
 *   tokens : [T].  A negative token is no token: its row of O is zero.  A token >= V is a mistake that only
 *            the device can see: its row of O is NaN, nothing is read out of bounds.
 *   table  : [V,D];  O : [T,D], the same dtype; product in fp32, rounded once.
 *   mult   : [T] fp32 (gene counts, say) or NULL (all ones).
 * T <= 2^31 - 1, 1 <= V <= 2^30, 1 <= D <= 65536 (else SPHATTN_ERR_SHAPE).
 */
int sphattn_embed_fwd(const void* tokens, int id_bytes, const void* table, const float* mult, void* O,
                      int T, int V, int D, float scale, int dtype, void* stream);

/*
 * Gradient of the whole table:  dtable[v,:] = scale * sum over t with tokens[t] == v of mult[t] * dO[t,:]
 * Every row of dtable is written (zeros where no token is v); tokens outside 0 .. V-1 add nothing.  Sums run in
 * fp32 in the order of t within pieces of the sorted tokens, the same in every run, and are rounded once.
 *   workspace : at least sphattn_embed_bwd_workspace_bytes(T, V, D) bytes (0 for sizes the call would reject),
 *               SPHATTN_ERR_WORKSPACE otherwise.
 */
size_t sphattn_embed_bwd_workspace_bytes(int T, int V, int D);
int sphattn_embed_bwd(const void* tokens, int id_bytes, const float* mult, const void* dO, void* dtable,
                      int T, int V, int D, float scale, int dtype,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * Cross entropy of a linear head over a vocabulary, without its logits in memory:
 *   l[t,v] = scale * X[t,:] . W[v,:]     lse[t] = log(sum over v of exp l[t,v])     losses[t] = lse[t] - l[t,targets[t]]
 *   X : [T,D], W : [V,D], targets : [T].  A negative target means that the row does not count: its loss is 0 and its
 *   gradients are zeros.  A target >= V is a mistake that only the device can see: the row's loss and lse are NaN, and so
 *   are the gradients that it takes part in.
 *   losses, lse : [T] fp32.  lse may be NULL.
 *   mean : one fp32, or NULL: the sum of the losses (reduction SPHATTN_LOSS_SUM) or their mean over the rows that
 *          count (SPHATTN_LOSS_MEAN; 0 if none does).  Not looked at with SPHATTN_LOSS_NONE.
 *   all_rows : 1: lse also of rows that do not count; 0: those rows cost nothing and get lse 0.
 * fp32 sums of exact products (SPHATTN_F32 with more than 64 rows: the factors to 2^-23 on average and 2^-22 at most, those
 * below 2^-29 of their row's largest element to 2^-51 of that; terms off by 3/4 2^-20 at most).  Infinite and NaN elements give
 * the logits that the sum gives.  T <= 2^20, 1 <= V <= 2^24, 1 <= D <= 65536
 * (SPHATTN_ERR_SHAPE); scale finite, reduction a sphattn_reduction (SPHATTN_ERR_VALUE).
 * Workspace sizes are 0 for sizes that the call would reject.
 */
typedef enum { SPHATTN_LOSS_NONE = 0, SPHATTN_LOSS_SUM = 1, SPHATTN_LOSS_MEAN = 2 } sphattn_reduction;

size_t sphattn_vocab_loss_workspace_bytes(int T, int V, int D, int dtype);
int sphattn_vocab_loss_fwd(const void* X, const void* W, const void* targets, int id_bytes,
                           float* losses, float* lse, float* mean,
                           int T, int V, int D, float scale, int reduction, int all_rows, int dtype,
                           void* workspace, size_t workspace_bytes, void* stream);

/*
 * Gradients of that:  G[t,v] = g[t] (exp(l[t,v] - lse[t]) - [v == targets[t]]) for rows that count, 0 for others
 *                     dX = scale * G W      dW = scale * G^T X
 *   lse   : [T], from the forward call.
 *   dloss : SPHATTN_LOSS_NONE: [T] fp32, g = dloss;  SUM: one fp32, g[t] = dloss;  MEAN: one fp32, g[t] = dloss / (number of
 *           rows that count).
 *   dX : [T,D], dW : [V,D], the dtype of X and W; either may be NULL (not wanted), not both.
 * G is formed a piece of the vocabulary at a time and rounded to the storage type; sums in fp32, the results rounded once.  fp16: G is
 * scaled by powers of two, so that it keeps the type's bits down to 2^-28 of a row's gradient and 2^-38 of that at the least; with
 * SPHATTN_LOSS_NONE in dW of the largest gradient of a row that counts.  (Where the rows' gradients differ by more than 2^4 it is formed
 * once for dX and once for dW.)  SPHATTN_F32: every factor keeps its 24 bits whatever
 * the others' sizes are, terms are off by 2^-24 at most.
 */
size_t sphattn_vocab_loss_bwd_workspace_bytes(int T, int V, int D, int dtype);
int sphattn_vocab_loss_bwd(const void* X, const void* W, const void* targets, int id_bytes,
                           const float* lse, const float* dloss, void* dX, void* dW,
                           int T, int V, int D, float scale, int reduction, int dtype,
                           void* workspace, size_t workspace_bytes, void* stream);

/*
 * Clipping of gradients by their common 2-norm:
 *   norm = sqrt(sum over all elements of all tensors of in^2)      out[i] = in[i] * min(1, max_norm / (norm + 1e-6))
 *   in, out : host arrays of n device pointers; out[i] may be in[i] (then it is not written where the factor
 *             is 1) and overlaps no other tensor (not checked).  Tensor i has size[i] >= 0 elements of type dtype[i],
 *             2^40 in all at most (SPHATTN_ERR_SHAPE).
 *   norm    : device, one fp32; written by the call.  Squares are added in fp64; a norm that is not
 *             finite gives a factor of 0 (infinite) or NaN, as the formula does.
 *   max_norm: >= 0 (SPHATTN_ERR_VALUE for negative ones and NaN).  n >= 0; the host arrays are read before the call returns.
 *   workspace : at least sphattn_clip_grads_workspace_bytes(n) bytes.
 * Two launches per 120 tensors.
 */
size_t sphattn_clip_grads_workspace_bytes(int n);
int sphattn_clip_grads(const void* const* in, void* const* out, const long long* size, const int* dtype, int n,
                       float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SPHATTN_TRAIN_H */
