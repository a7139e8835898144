// What the host code of the products that are consumed in place shares: the choice of their tiles, their arguments, and the gradient of a loss over
// a vocabulary.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <functional>

#include "../../include/gensor_fused.h"
#include "fused_registry.hpp"
#include "host_common.hpp"

namespace gensor {

inline bool valid_dtype(int d) { return d == GENSOR_F32 || d == GENSOR_F16 || d == GENSOR_BF16; }
inline int size_of(int d) { return d == GENSOR_F32 ? 4 : 2; }
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline GemmView product_view(int in_dtype, int out_dtype, int64_t M, int64_t N, int64_t K, int asrc, int bsrc, int64_t batch = 1) {
  GemmView v;
  std::memset(&v, 0, sizeof(v));
  v.M = M; v.N = N; v.K = K; v.batch = batch;
  v.in_dtype = in_dtype; v.out_dtype = out_dtype; v.esize = size_of(in_dtype); v.osize = size_of(out_dtype);
  v.asrc = asrc; v.bsrc = bsrc;
  return v;
}

struct FusedChoice {
  const FusedDesc* f;
  int split;
  size_t bytes;
  double us;
};

// The cheapest tile with this end by the cost model, of those that reach the operands' rows and fit the room for partial tiles.
gensor_status choose(const GemmView& v, int kind, bool vec_ok, const LeadingDims& ld, size_t room, FusedChoice* out);

// `panel`: tile rows that are walked together, column by column (L2 reuse).
inline void tiles_of(FusedArgs* a, const GemmView& v, const FusedChoice& c, int64_t M, int64_t N, int panel = 4) {
  const InstanceDesc& d = c.f->d;
  a->tiles_m = (int32_t)((M + d.bm - 1) / d.bm);
  const int bn = a->narrow ? 192 : d.bn;
  a->tiles_n = (int32_t)((N + bn - 1) / bn);
  a->batch = (int32_t)v.batch;
  a->panel = std::min(panel, std::max(1, a->tiles_m));
  a->lds_stages = d.stages;
}

// The part of the arguments that every product shares.  C's rows are stored past the caches unless a large output's rows do
// not start on cache lines (as gensor_gemm does).
inline FusedArgs product_args(const GemmView& v, const void* A, int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc, float alpha) {
  FusedArgs a;
  std::memset(&a, 0, sizeof(a));
  a.A = A; a.B = B; a.C = C;
  a.M = (int32_t)v.M; a.N = (int32_t)v.N; a.K = (int32_t)v.K;
  a.lda = lda; a.ldb = ldb; a.ldc = ldc;
  a.alpha = alpha;
  a.store_m = a.M; a.store_n = a.N;
  a.split = 1;
  const int64_t c_bytes = v.batch * v.M * v.N * v.osize;
  a.through = !((ldc * v.osize) % 128 != 0 && c_bytes > (v.osize == 2 ? 32ll : 64ll) * 1024 * 1024);
  return a;
}

// Are the columns 2j and 2j + 1 of a 16-bit matrix one aligned dword?
inline bool pairs(const void* p, int64_t ld, int64_t N, int osize) { return osize == 2 && N % 2 == 0 && ld % 2 == 0 && aligned(p, 4); }

// Nothing leaves a C entry as an exception (the host's containers may run out of memory).
template <typename F>
inline gensor_status guarded(F&& body) {
  try {
    return body();
  } catch (...) {
    return GENSOR_ERR_DEVICE;
  }
}

// The kernels number rows and columns to the end of the last tile in 32 bits.
inline bool extents_fit(const GemmView& v) { return v.M <= INT32_MAX - 256 && v.N <= INT32_MAX - 256 && v.K <= INT32_MAX - 256; }

inline gensor_status launched(hipError_t e) { return e == hipSuccess ? GENSOR_OK : GENSOR_ERR_DEVICE; }

inline size_t usable_room(const void* workspace, size_t bytes) { return workspace && aligned(workspace, 256) ? bytes : 0; }

inline size_t round_up(size_t n, size_t to) { return (n + to - 1) / to * to; }

// The gradient of a loss over a vocabulary, dX = G W and dW = G^T X, a piece of the vocabulary at a time (gensor_xent_backward says how).  What G
// is, the loss says: `prepare` runs once before the pieces (scales: the factor of G and its inverse, to be written; null in fp32),
// `piece` puts G of the piece into a.C: the arguments of the product with the vocabulary's rows as rows [a.row_first, a.row_first + a.M) are ready, and the tiles.
struct VocabularyLoss {
  std::function<hipError_t(float* scales, hipStream_t st)> prepare;
  std::function<hipError_t(FusedArgs& a, const FusedDesc& tile, hipStream_t st)> piece;
};
gensor_status vocabulary_gradient(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx, const void* W, int64_t ldw,
                                  const VocabularyLoss& loss, void* dX, int64_t lddx, void* dW, int64_t lddw, void* workspace, size_t workspace_bytes, hipStream_t s);
gensor_status check_xent(gensor_dtype dtype, int64_t T, int64_t V, int64_t D);
GemmView prob_view(int dtype, int64_t rows, int64_t T, int64_t D);

}  // namespace gensor
