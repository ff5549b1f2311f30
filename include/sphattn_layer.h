/*
 * sphattn -- what a layer has around the attention of sphattn.h, C ABI: the norms and rotations of its queries and
 * keys, and the gated feed-forward product behind it, with their gradients.
 *
 * Conventions are those of sphattn_train.h: device pointers owned by the caller, nothing allocated, no state, work
 * enqueued on `stream` without synchronising, one of sphattn.h's return codes; dtype SPHATTN_F32, SPHATTN_BF16 or
 * SPHATTN_F16; pointers aligned to one element, workspaces to 16 bytes.  Calls that share a workspace must be ordered.
 * Results do not depend on the order in which workgroups run: no float is added atomically.
 */
#ifndef SPHATTN_LAYER_H
#define SPHATTN_LAYER_H

#include "sphattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Rows of d neighbouring elements by sequence, token and head: element i of (b, n, h) is data[b batch + n token + h head + i].
 * Strides are in elements and not negative.  A tensor that is read may have any (0 where one row serves many); one that is
 * written has a place of its own for every row (SPHATTN_ERR_ALIAS where its strides say otherwise).
 */
typedef struct { void* data; long long batch, token, head; } sphattn_heads;

/* Positions of the tokens, and how fast each pair of dimensions turns with them. */
typedef struct {
    const void* positions;       /* axis a, sequence b, token n: positions[a axis + b batch + n]; NULL: nothing is rotated */
    int id_bytes;                /* 4 (int32) or 8 (int64) */
    long long axis, batch;       /* strides in elements, not negative */
    const float* inv_freq;       /* [d/2], radians per position */
    int axes;                    /* 1 to 3 */
    int sections[3];             /* frequencies that go by the first, second and third axis, in order; together d/2 */
    int interleaved;             /* 0: dimension i turns with i + d/2, 1: 2i with 2i + 1 */
} sphattn_rotary;

/*
 * Queries and keys of a projection, head by head:
 *   y = x w / sqrt(mean(x^2) + eps)  (norm 1)  or  x w  (norm 0)
 *   angle_i = position[axis of i] inv_freq[i]       (a, b) -> (a cos - b sin, b cos + a sin) for each pair of dimensions
 *   Xq, Xk : [B,N,Hq,d] and [B,N,Hk,d] by strides; Xk may be NULL (Hk then 0).
 *   wq, wk : [d], the type of X, or NULL (ones).
 *   Q, K   : where the rows go, by strides: [B,Hq,N,d] for the attention, or a place in a cache.  They overlap no input
 *            (SPHATTN_ERR_ALIAS) and each other nowhere (not checked: both may lie in one buffer).  What is between the rows is not touched.
 *   rotary : NULL: nothing is rotated.  Turns (position inv_freq / 2 pi) are formed in fp64, off by 2^-51 of themselves, their fraction is rounded to fp32: at 2^31 and a radian
 *            per position 2^-22 of a turn, larger frequencies in proportion.
 * In fp32, rounded once, whatever the size of a row's elements.  d 64 or 128 (SPHATTN_ERR_HEAD_DIM); B, N >= 0 (0: nothing is done), B N <= 2^31 - 1, Hq >= 1, Hk >= 0, Hq + Hk <= 65536, sections
 * as said (SPHATTN_ERR_SHAPE); eps >= 0 and finite, norm 0 or 1 (SPHATTN_ERR_VALUE).
 */
int sphattn_head_norm_rotary_fwd(const sphattn_heads* Xq, const sphattn_heads* Xk, const void* wq, const void* wk, const sphattn_heads* Q, const sphattn_heads* K,
                                 const sphattn_rotary* rotary, int B, int N, int Hq, int Hk, int d, int norm, float eps, int dtype, void* stream);

/*
 * Gradients of that: dQ, dK (by strides) -> dXq, dXk (by strides; NULL: not wanted) and dwq, dwk ([d], the type of w; NULL: not wanted; all zeros
 * where B N is 0).  At least one is wanted (SPHATTN_ERR_NULL).  dwq sums over all sequences, tokens and query heads, in fp32.
 *   workspace : at least sphattn_head_norm_rotary_bwd_workspace_bytes(d) bytes (0 for other d); not needed (may be NULL) where neither dwq nor
 *               dwk is wanted.
 */
size_t sphattn_head_norm_rotary_bwd_workspace_bytes(int d);
int sphattn_head_norm_rotary_bwd(const sphattn_heads* Xq, const sphattn_heads* Xk, const void* wq, const void* wk, const sphattn_heads* dQ, const sphattn_heads* dK,
                                 const sphattn_heads* dXq, const sphattn_heads* dXk, void* dwq, void* dwk, const sphattn_rotary* rotary,
                                 int B, int N, int Hq, int Hk, int d, int norm, float eps, int dtype, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The gated feed-forward product of a layer:  H = act(X Wg^T) * (X Wu^T)
 *   X : [T,D], Wg, Wu : [F,D], H : [T,F], contiguous, of one type.  Sums and act in fp32, rounded once.
 *   act: silu a / (1 + e^-a), gelu a Phi(a) (with the normal distribution's Phi), relu max(a, 0).
 * SPHATTN_F32 with more than 64 rows: the factors to 2^-23 on average and 2^-22 at most, those below 2^-29 of their row's largest element to 2^-51 of
 * that; terms off by 3/4 2^-20 at most.  T <= 2^20 (0: nothing is done), 1 <= D <= 65536, 1 <= F <= 2^18, T F <= 2^36 (SPHATTN_ERR_SHAPE); gate a sphattn_gate
 * (SPHATTN_ERR_VALUE).  Outputs overlap neither each other nor inputs nor the workspace (SPHATTN_ERR_ALIAS).
 *   workspace : at least sphattn_gated_ffn_workspace_bytes(T, D, F, dtype) bytes (0 for sizes that the call would reject, and where it needs
 *               none: it may be NULL then).
 */
typedef enum { SPHATTN_GATE_SILU = 0, SPHATTN_GATE_GELU = 1, SPHATTN_GATE_RELU = 2 } sphattn_gate;

size_t sphattn_gated_ffn_workspace_bytes(int T, int D, int F, int dtype);
int sphattn_gated_ffn_fwd(const void* X, const void* Wg, const void* Wu, void* H, int T, int D, int F, int gate, int dtype,
                          void* workspace, size_t workspace_bytes, void* stream);

/*
 * Gradients of that, from its inputs alone (A = X Wg^T and U = X Wu^T are formed again):
 *   dA = dH U act'(A)    dB = dH act(A)    dX = dA Wg + dB Wu    dWg = dA^T X    dWu = dB^T X        (relu: act' is 1 where A is greater than 0, else 0, as a sum in fp64 has it)
 *   dH : [T,F].  dX : [T,D], dWg, dWu : [F,D]; each may be NULL (not wanted), not all (SPHATTN_ERR_NULL; T = 0: all).  T = 0: dWg and dWu are zeros.
 * dA and dB are rounded once to the storage type (up to 2^18 of them to twice its bits; SPHATTN_F32: not; every factor of the sums keeps its 24 bits, terms are off by 2^-24 at
 * most), sums in fp32, the results rounded once.  fp16: dA and dB are scaled by powers of two, for dX by row and for dW by column, from what
 * the norms of X's and W's rows and the largest dH of the row or column allow at most: values down to 2^-27 of that keep the type's bits.
 * Where they have more than 16 bits an infinite element of dA, dB, X or W may make NaN of a sum that it would make infinite.
 */
size_t sphattn_gated_ffn_bwd_workspace_bytes(int T, int D, int F, int dtype);
int sphattn_gated_ffn_bwd(const void* X, const void* Wg, const void* Wu, const void* dH, void* dX, void* dWg, void* dWu, int T, int D, int F,
                          int gate, int dtype, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SPHATTN_LAYER_H */
