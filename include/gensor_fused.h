/*
 * gensor_fused.h -- products that are consumed where they are produced: C ABI, beside gensor.h, whose conventions, types and
 * status codes hold here.
 *
 * These operators end a product in the kernel that computes it: a layer's bias, activation and residual, the gradient through
 * the activation, products grouped by expert, and the cross entropy of a projection onto a large vocabulary.  They choose
 * their tiles by the same cost model (per shape, remembered; no gensor_schedule).  Products and sums are carried in fp32
 * and rounded once, where a result is stored.  Types are those of gensor_gemm: operands of in_dtype, results of out_dtype, which is
 * GENSOR_F32 or in_dtype.  Rows may start anywhere; operands on 16-byte boundaries with rows of whole 16-byte vectors run the fastest
 * tiles, and 16-bit results (and what is read and kept beside them) on dword boundaries with even rows are stored in whole lines.  UNSUPPORTED: leading
 * dimensions so large that no tile's rows stay within 32-bit offsets (32-row tiles reach 2^31 / 33 bytes), or extents above
 * INT32_MAX - 256.
 */
#ifndef GENSOR_FUSED_H
#define GENSOR_FUSED_H

#include "gensor.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  GENSOR_ACT_NONE = 0,
  GENSOR_ACT_RELU = 1,          /* max(z, 0) (NaN stays) */
  GENSOR_ACT_GELU = 2,          /* tanh form: 0.5 z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) */
  GENSOR_ACT_SILU = 3           /* z / (1 + exp(-z)) */
} gensor_act;

/*
 * What a product ends in.  grad = 0:
 *     Z = alpha * op(A) * op(B) + bias,   C = act(Z) + residual
 * bias has one value of in_dtype per column (per group and column for grouped products: [groups][N]); preact, if not null, receives
 * Z in out_dtype (as the gradient needs it); residual is of out_dtype and may be C itself with the same leading dimension.
 * grad = 1, the gradient through the activation:
 *     C = (alpha * op(A) * op(B)) * act'(preact)
 * with preact of out_dtype read (it may be C itself with the same leading dimension), no bias and no residual.  act' of relu is 0 at 0.
 */
typedef struct {
  int32_t act;                  /* gensor_act */
  int32_t grad;                 /* 0 or 1 */
  const void* bias;             /* or NULL */
  void* preact;                 /* or NULL (grad = 1: required) */
  int64_t ld_preact;
  const void* residual;         /* or NULL */
  int64_t ld_residual;
} gensor_epilogue;

/* The product of gensor_gemm (p->op = GENSOR_OP_GEMM) with an epilogue; e == NULL: C = alpha * op(A) * op(B).  transA = 1 together with
 * transB = 1 is UNSUPPORTED.  `workspace` holds the partial tiles of split products (256-byte aligned,
 * gensor_gemm_fused_workspace_bytes(p) for the best choice); with less, or none, the best choice that needs no more is taken. */
gensor_status gensor_gemm_fused(const gensor_problem* p, const gensor_epilogue* e, float alpha,
                                const void* A, int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc,
                                void* workspace, size_t workspace_bytes, void* hip_stream);
size_t gensor_gemm_fused_workspace_bytes(const gensor_problem* p);

/*
 * Products grouped by expert, ragged: p->op = GENSOR_OP_BMM, p->batch = groups, p->M = the rows of all groups together (0 is no
 * error), transA = 0.  Rows are sorted by group: group g owns rows [offsets[g], offsets[g+1]) of A and C, where `offsets` are
 * groups + 1 non-decreasing int32 in DEVICE memory; any group may be empty.  The host never reads them and never waits for them.
 * Rows in front of offsets[0] or behind offsets[groups] belong to no group: they are not read and not written.  Offsets outside
 * [0, p->M] or decreasing ones are cut to what exists: results of such calls are unspecified, no access is out of bounds.
 *     C[r] = epilogue(alpha * A[r] * op(B[g]))   for the rows r of group g
 * B[g] is strideB elements behind B[g-1] (0: all groups share it), stored [K][N], or [N][K] if transB.
 * The gradient of A is the same call with N and K and transB exchanged.
 */
gensor_status gensor_grouped_gemm(const gensor_problem* p, const int32_t* offsets, const gensor_epilogue* e, float alpha,
                                  const void* A, int64_t lda, const void* B, int64_t ldb, int64_t strideB,
                                  void* C, int64_t ldc, void* hip_stream);

/* The gradient of B for the same p: dW[g] = A_g^T * dY_g over the rows of g, stored like B ([K][N], or [N][K] if transB), of out_dtype, zeros
 * for an empty group.  A is [rows][K], dY [rows][N], both of in_dtype; dW[g] is stride_dw elements behind dW[g-1]. */
gensor_status gensor_grouped_wgrad(const gensor_problem* p, const int32_t* offsets, const void* A, int64_t lda,
                                   const void* dY, int64_t lddy, void* dW, int64_t lddw, int64_t stride_dw, void* hip_stream);

/* The gradient of a bias: db[g][n] = sum over the rows r of group g of dY[r][n].  offsets as above, or NULL with groups = 1 for all rows.
 * db is [groups][N] of out_dtype (zeros for an empty group).  The workspace (4-byte aligned) holds partial sums;
 * with less than gensor_bias_grad_workspace_bytes fewer workgroups share the rows.  The order of the sums is fixed. */
gensor_status gensor_bias_grad(gensor_dtype in_dtype, gensor_dtype out_dtype, int64_t groups, int64_t rows, int64_t N,
                               const void* dY, int64_t ld, const int32_t* offsets, void* db,
                               void* workspace, size_t workspace_bytes, void* hip_stream);
size_t gensor_bias_grad_workspace_bytes(gensor_dtype in_dtype, int64_t groups, int64_t rows, int64_t N);

/*
 * Softmax cross entropy of the logits z = X * W^T, which are never stored: X is [T][D] (tokens), W [V][D] (vocabulary), both of
 * `dtype`, targets int64 on the device.
 *     lse[t] = log sum_v exp(z[t][v]),   loss[t] = lse[t] - z[t][targets[t]]
 * in fp32; loss[t] = 0 where targets[t] == ignore_index, NaN where a target is neither that nor in [0, V).  loss or lse may be NULL (targets
 * too, without loss).  The workspace (256-byte aligned) holds a maximum and a sum per token and slab of the vocabulary.  What
 * gensor_xent_workspace_bytes(..., 0) asks for serves any leading dimensions; with less, or where rows are too far apart for the tile it is
 * meant for, the vocabulary is taken in pieces, a pair of launches each.  WORKSPACE if not even one row of tiles' slabs fit beside the sums so far.
 */
gensor_status gensor_xent_forward(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx,
                                  const void* W, int64_t ldw, const int64_t* targets, int64_t ignore_index,
                                  float* loss, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Its gradient: with G[t][v] = dloss[t] * (exp(z[t][v] - lse[t]) - (v == targets[t])), zero for tokens whose target is ignore_index
 * or outside [0, V), whatever their logits, their lse and their dloss are,
 *     dX = G * W,   dW = G^T * X
 * in `dtype`; dX or dW may be NULL.  (A row of X that is not finite reaches dW as zero times it.)  lse is the forward's, dloss (fp32, device) the
 * gradient of each token's loss.  The logits are computed again, a piece of the vocabulary at a time: G of a piece lies in the workspace in
 * `dtype` (16-bit types: scaled so that the largest |dloss| of the tokens that count is 2^15, undone in fp32), and dX is
 * summed over the pieces in fp32.  gensor_xent_workspace_bytes(..., 1) asks for 256 MiB of G at most (all of it, where that is less), dX's sums
 * and partial tiles.  With less workspace the pieces are smaller, down to 256 entries; WORKSPACE if not even those fit.  (4096 tokens over 50257
 * entries of width 768 in bf16, whose logits are 393 MiB: 306 MiB 866 us, 192 1082, 128 1259, 64 1721.)
 */
gensor_status gensor_xent_backward(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx,
                                   const void* W, int64_t ldw, const int64_t* targets, int64_t ignore_index,
                                   const float* lse, const float* dloss, void* dX, int64_t lddx, void* dW, int64_t lddw,
                                   void* workspace, size_t workspace_bytes, void* hip_stream);
size_t gensor_xent_workspace_bytes(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, int32_t backward);

#ifdef __cplusplus
}
#endif
#endif /* GENSOR_FUSED_H */
