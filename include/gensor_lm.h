/*
 * gensor_lm.h -- a language model's gated layers, the scores of its vocabulary, and learning from a teacher: C ABI, beside gensor.h and
 * gensor_fused.h, whose conventions, types and status codes hold here.
 *
 * Products and sums are carried in fp32 and rounded once, where a result is stored.  Tiles are chosen by the cost model (per shape, remembered).
 * Operands on 16-byte boundaries with rows of whole 16-byte vectors run the fastest tiles; rows may start anywhere.  UNSUPPORTED: leading
 * dimensions or distances so large that no tile's rows stay within 32-bit offsets, or extents above INT32_MAX - 256.
 */
#ifndef GENSOR_LM_H
#define GENSOR_LM_H

#include "gensor_fused.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A gated layer's first half: p is the product of gensor_gemm (p->op = GENSOR_OP_GEMM, transA = 0) with either of two matrices B,
 *     G = alpha * A * op(B0) + bias0,   U = alpha * A * op(B1) + bias1,   C = act(G) * U
 * B1 lies strideB elements behind B0, both [K][N], or [N][K] if transB, with the leading dimension ldb, in one allocation: all memory from B0's
 * first to B1's last element must be there.  One matrix [K][2N] of both is ldb = 2N, strideB = N; [2N][K] is strideB = N * ldb.  bias is [2][N] of
 * in_dtype, or NULL.  preact, if not null, receives G, and U stride_preact elements behind it, in out_dtype, as the gradient needs them.  C, G and U
 * must not overlap (unless side by side in one matrix's rows).
 */
gensor_status gensor_gated_gemm(const gensor_problem* p, int32_t act, float alpha, const void* A, int64_t lda,
                                const void* B, int64_t ldb, int64_t strideB, const void* bias, void* C, int64_t ldc,
                                void* preact, int64_t ld_preact, int64_t stride_preact, void* hip_stream);

/*
 * Its gradient, at the end of the product that leads to the layer's result (p: transA = 0; a block's: A the gradient of its output, B its second
 * projection):
 *     D = alpha * A * op(B),   dG = D * U * act'(G),   dU = D * act(G),   H = act(G) * U
 * G and U as gensor_gated_gemm left them, in out_dtype; dG, and dU stride_dpreact elements behind it, of out_dtype, may be G and U themselves
 * with the same leading dimension and distance.  H (of out_dtype) is the layer's result again, which the second projection's gradient needs; NULL: not wanted.
 * The other gradients are plain products: of the input dG * B0^T + dU * B1^T (one product where the two lie in one matrix), of the weights A^T * dG and
 * A^T * dU.  act' of relu is 0 at 0.
 */
gensor_status gensor_gated_act_grad(const gensor_problem* p, int32_t act, float alpha, const void* A, int64_t lda, const void* B, int64_t ldb,
                                    const void* preact, int64_t ld_preact, int64_t stride_preact,
                                    void* dpreact, int64_t ld_dpreact, int64_t stride_dpreact, void* H, int64_t ldh, void* hip_stream);

/*
 * Scores of the logits z = scale * X * W^T, which are not kept: X [T][D] (tokens) and W [V][D] (vocabulary) of `dtype`; scale > 0, finite, is the
 * inverse of a temperature.  Each of the outputs may be NULL, not all of them:
 *     logprob[t] = z[t][targets[t]] - lse[t]           0 where targets[t] == ignore_index, NaN where it is neither that nor in [0, V)
 *     lse[t] = log sum_v exp(z[t][v])
 *     entropy[t] = - sum_v p log p,  p = exp(z[t][v] - lse[t])
 *     top_index[t][j], top_logprob[t][j]               the `top` largest logits' entries and their log probabilities, falling; of equal
 *                                                      logits the lowest entry first
 * top is 0 or up to GENSOR_TOP_MAX and V; top_index (int64) and top_logprob (fp32) are [T][top], and both are wanted where top > 0.  targets (int64) are
 * wanted with logprob.  A NaN among a token's logits makes its log probabilities and entropy NaN; it is no alternative, and entry -1 stands where fewer than
 * `top` others are.  (An infinite largest logit: lse is that, what is a difference of infinities NaN.)
 * The workspace (256-byte aligned) holds, beside sums, the logits of a piece of the vocabulary that may be among the largest.
 * gensor_logprobs_workspace_bytes asks for what pieces of 384 MiB (or of one row of tiles, where many tokens make that more) want, for any leading
 * dimensions; with less the pieces are smaller.  What it holds beforehand does not matter.
 * WORKSPACE if not even one row of tiles fits.
 */
#define GENSOR_TOP_MAX 64
gensor_status gensor_logprobs(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx,
                              const void* W, int64_t ldw, float scale, const int64_t* targets, int64_t ignore_index,
                              float* logprob, float* lse, float* entropy, int32_t top, int64_t* top_index, float* top_logprob,
                              void* workspace, size_t workspace_bytes, void* hip_stream);
size_t gensor_logprobs_workspace_bytes(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, int32_t top);

/*
 * The distillation loss against a teacher's top entries: index [T][k] (int64, device) names entries of the vocabulary, -1 none (what stands
 * beside it is not read as a number), teacher [T][k] (fp32) their log probabilities.  With z and lse as above,
 *     normalize = 1:  p = softmax over the token's entries of scale * teacher   (logits will do, too)
 *     normalize = 0:  p = exp(teacher)
 *     loss[t] = sum_j p_j (log p_j - z[t][index_j] + lse[t])
 * A teacher's log probability of -inf is a probability of zero.  A token without entries, or with probabilities of zero only, has a loss of 0; an entry below -1
 * or not below V makes it NaN.  An entry that is named twice counts twice.  loss or lse (fp32) may be NULL.  1 <= k <= GENSOR_TEACHER_MAX.
 */
#define GENSOR_TEACHER_MAX 256
gensor_status gensor_distill_forward(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx,
                                     const void* W, int64_t ldw, float scale, int32_t k, const int64_t* index, const float* teacher, int32_t normalize,
                                     float* loss, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Its gradient: with G[t][v] = dloss[t] * scale * (P exp(z[t][v] - lse[t]) - sum of p_j over index_j == v),  P = sum_j p_j,
 *     dX = G * W,   dW = G^T * X
 * in `dtype`; dX or dW may be NULL.  G is zero for tokens whose loss is 0 for want of entries, whose loss is NaN for an entry out of range, and whose dloss is
 * zero, whatever their logits and lse are.  lse is the forward's, dloss (fp32, device) the gradient of each token's loss.  Pieces, G's scale in 16 bits
 * (to which it is rounded, as the products' operand) and room are as in gensor_xent_backward; gensor_distill_workspace_bytes(..., 1) asks for that and
 * T (8 k + 4) bytes more, rounded up to 256.
 */
gensor_status gensor_distill_backward(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx,
                                      const void* W, int64_t ldw, float scale, int32_t k, const int64_t* index, const float* teacher, int32_t normalize,
                                      const float* lse, const float* dloss, void* dX, int64_t lddx, void* dW, int64_t lddw,
                                      void* workspace, size_t workspace_bytes, void* hip_stream);
size_t gensor_distill_workspace_bytes(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, int32_t k, int32_t backward);

#ifdef __cplusplus
}
#endif
#endif /* GENSOR_LM_H */
