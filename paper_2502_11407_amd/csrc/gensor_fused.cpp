// C ABI of the products that are consumed in place: gensor_gemm_fused, gensor_grouped_gemm, gensor_grouped_wgrad,
// gensor_bias_grad, gensor_xent_forward and gensor_xent_backward.  Argument validation, the choice of the tile, the launches and the
// small kernels between the products.  No device memory is allocated here.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <array>
#include <cstring>
#include <map>
#include <mutex>
#include <vector>

#include "../../include/gensor_fused.h"
#include "fused_registry.hpp"
#include "host_common.hpp"

using namespace gensor;

namespace {

bool valid_dtype(int d) { return d == GENSOR_F32 || d == GENSOR_F16 || d == GENSOR_BF16; }
int size_of(int d) { return d == GENSOR_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

GemmView product_view(int in_dtype, int out_dtype, int64_t M, int64_t N, int64_t K, int asrc, int bsrc, int64_t batch = 1) {
  GemmView v;
  std::memset(&v, 0, sizeof(v));
  v.M = M; v.N = N; v.K = K; v.batch = batch;
  v.in_dtype = in_dtype; v.out_dtype = out_dtype; v.esize = size_of(in_dtype); v.osize = size_of(out_dtype);
  v.asrc = asrc; v.bsrc = bsrc;
  return v;
}

// ------------------------------------------------------------------------------------
// The tile: the cheapest by the cost model of those that exist with this end, reach the operands' rows and fit the room for partial
// tiles.  Remembered per shape.
// ------------------------------------------------------------------------------------
struct FusedChoice {
  const FusedDesc* f;
  int split;
  size_t bytes;
  double us;
};
std::mutex g_choice_mutex;
std::map<std::array<int64_t, 14>, std::vector<FusedChoice>> g_choices;
const size_t kChoiceLimit = 4096;
// (five parts: 48 tiles of 256x256, a gradient of 4096 x 768 over a piece of the vocabulary, fill 240 of 256 units)
const int kSplits[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16};

// The cost model's time.  A group's tiles of a product over ragged rows take as long as its rows are many, and groups are rarely even: a launch
// is no shorter than one group of three times the mean's rows alone.  (8 groups of 2048 rows on average, the largest 5000, 768 x 3072 each:
// 256x256 tiles 121 us, 256x128 103; 32 groups of 512: 125 and 149.)
// (An unsplit 256x256 tile is priced as 192-column ones where narrow_tiles() says so, for the grouped, logit and probability ends too, which have no such
// form.  At the price of the wide form 1.2 % of the choices over drawn shapes change, to smaller tiles: 53 of them took 0.80 to 1.35 of the
// time, in the geometric mean 1.004.)
double tile_price(const FusedDesc& f, const GemmView& v, int kind, int split) {
  const double us = fused_price(f.d, v, split);
  if (kind != FUSED_DEPTH || us <= 0 || v.batch == 1) return us;
  GemmView one = v;
  one.batch = 1;
  one.K = std::min<int64_t>(3 * v.K, INT32_MAX - 256);
  return std::max(us, fused_price(f.d, one, 1));
}

// Can one launch have all of the product's tiles?  (Split tiles add less than sixteen rounds.)
bool tiles_fit(const InstanceDesc& d, const GemmView& v, int kind) {
  const int64_t bn = d.alternate() && kind == FUSED_LINEAR ? 192 : d.bn;
  const double tiles = (double)((v.M + d.bm - 1) / d.bm) * (double)v.batch * (double)((v.N + bn - 1) / bn);
  // (the logits' workgroups stay: a fixed number of them, each of which counts one round beyond its last tile)
  if (kind == FUSED_LSE && d.alternate()) return tiles <= INT32_MAX - gensor_hw_mi355x()->compute_units;
  if (kind == FUSED_ROWS) return true;                                       // any number of launches
  return launch_fits(tiles + 16 * gensor_hw_mi355x()->compute_units, d.threads);
}

gensor_status choose(const GemmView& v, int kind, bool vec_ok, const LeadingDims& ld, size_t room, FusedChoice* out) {
  const std::array<int64_t, 14> key = {kind, v.in_dtype, v.out_dtype, v.asrc, v.bsrc, vec_ok, v.M, v.N, v.K, v.batch, ld.a, ld.b, ld.c, 0};
  std::lock_guard<std::mutex> lock(g_choice_mutex);
  auto it = g_choices.find(key);
  if (it == g_choices.end()) {
    std::vector<FusedChoice> all;
    for (int i = 0; i < g_num_fused; ++i) {
      const FusedDesc& f = g_fused[i];
      if (!f.launch[kind] || !instance_serves(f.d, v) || (f.d.vec && !vec_ok) || !offsets_fit(f.d, v, ld) || !tiles_fit(f.d, v, kind)) continue;
      if (f.d.direct && !f.d.any_k() && (kind == FUSED_DEPTH || v.K % f.d.bk != 0)) continue;
      for (int split : kSplits) {
        if (split > 1 && (kind != FUSED_LINEAR || (v.K + f.d.bk - 1) / f.d.bk < split)) break;
        const double us = tile_price(f, v, kind, split);
        if (us <= 0) continue;
        const SplitPlan sp = split_plan(f.d, v, split, 0);
        if (split > 1 && sp.split == 1) continue;
        all.push_back({&f, split, sp.bytes, us});
      }
    }
    std::stable_sort(all.begin(), all.end(), [](const FusedChoice& a, const FusedChoice& b) { return a.us < b.us; });
    std::vector<FusedChoice> kept;           // in order of price, of strictly falling room
    for (const FusedChoice& c : all)
      if (kept.empty() || c.bytes < kept.back().bytes) kept.push_back(c);
    if (g_choices.size() >= kChoiceLimit) g_choices.clear();
    it = g_choices.emplace(key, std::move(kept)).first;
  }
  for (const FusedChoice& c : it->second)
    if (c.bytes <= room) { *out = c; return GENSOR_OK; }
  return GENSOR_ERR_UNSUPPORTED;
}

// `panel`: tile rows that are walked together, column by column (L2 reuse).
void tiles_of(FusedArgs* a, const GemmView& v, const FusedChoice& c, int64_t M, int64_t N, int panel = 4) {
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
FusedArgs product_args(const GemmView& v, const void* A, int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc, float alpha) {
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
bool pairs(const void* p, int64_t ld, int64_t N, int osize) { return osize == 2 && N % 2 == 0 && ld % 2 == 0 && aligned(p, 4); }

// Nothing leaves a C entry as an exception (the host's containers may run out of memory).
template <typename F>
gensor_status guarded(F&& body) {
  try {
    return body();
  } catch (...) {
    return GENSOR_ERR_DEVICE;
  }
}

// The kernels number rows and columns to the end of the last tile in 32 bits.
bool extents_fit(const GemmView& v) { return v.M <= INT32_MAX - 256 && v.N <= INT32_MAX - 256 && v.K <= INT32_MAX - 256; }

gensor_status launched(hipError_t e) { return e == hipSuccess ? GENSOR_OK : GENSOR_ERR_DEVICE; }

template <typename T, typename OutT>
hipError_t launch_reduce(const FusedArgs& a, const InstanceDesc& d, unsigned blocks, hipStream_t st) {
  hipLaunchKernelGGL((fused_split_reduce<T, OutT>), dim3(blocks), dim3(256), 0, st, a, d.bm, d.bn, d.wm, d.wn, d.mb);
  return hipGetLastError();
}

// One product with the linear end: whole tiles, or split ones and the launch that adds them up.
gensor_status run_linear(FusedArgs& a, const GemmView& v, const FusedChoice& c, void* workspace, hipStream_t st, int panel = 4) {
  const InstanceDesc& d = c.f->d;
  const SplitPlan sp = split_plan(d, v, c.split, 0);
  a.narrow = d.alternate() && sp.split == 1 && narrow_tiles(v, gensor_hw_mi355x()->compute_units);
  tiles_of(&a, v, c, v.M, v.N, panel);
  a.split = sp.split;
  a.whole = sp.split == 1 ? a.tiles_m * a.tiles_n : (int32_t)sp.whole;
  if (sp.split == 1) return launched(c.f->launch[FUSED_LINEAR](a, st));
  a.partials = (float*)workspace;
  const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n - a.whole, blocks = tiles * (d.bm * d.bn / 4) / 256;
  hipError_t e = c.f->launch[FUSED_LINEAR_SPLIT](a, st);
  if (e != hipSuccess) return GENSOR_ERR_DEVICE;
  const unsigned n = (unsigned)blocks;
  if (v.in_dtype == GENSOR_F32) e = launch_reduce<f32_t, f32_t>(a, d, n, st);
  else if (v.in_dtype == GENSOR_F16) e = v.osize == 4 ? launch_reduce<f16_t, f32_t>(a, d, n, st) : launch_reduce<f16_t, f16_t>(a, d, n, st);
  else e = v.osize == 4 ? launch_reduce<bf16_t, f32_t>(a, d, n, st) : launch_reduce<bf16_t, bf16_t>(a, d, n, st);
  return launched(e);
}

size_t usable_room(const void* workspace, size_t bytes) { return workspace && aligned(workspace, 256) ? bytes : 0; }

// The epilogue's arguments against the product's extents.
gensor_status check_epilogue(const gensor_epilogue* e, const GemmView& v, const void* C) {
  if (!e) return GENSOR_OK;
  if (e->act < GENSOR_ACT_NONE || e->act > GENSOR_ACT_SILU || (e->grad != 0 && e->grad != 1)) return GENSOR_ERR_INVALID_ARG;
  if (e->preact && e->ld_preact < v.N) return GENSOR_ERR_INVALID_ARG;
  if (e->residual && e->ld_residual < v.N) return GENSOR_ERR_INVALID_ARG;
  if (e->grad && (!e->preact || e->bias || e->residual)) return GENSOR_ERR_INVALID_ARG;
  if (!e->grad && e->preact && e->preact == C) return GENSOR_ERR_INVALID_ARG;
  return GENSOR_OK;
}

void set_epilogue(FusedArgs* a, const gensor_epilogue* e, const GemmView& v, LeadingDims* ld) {
  a->paired = pairs(a->C, a->ldc, v.N, v.osize);
  if (!e) return;
  a->act = e->act;
  a->grad = e->grad;
  a->bias = e->bias;
  a->preact = e->preact;
  a->residual = e->residual;
  a->ld_preact = e->ld_preact;
  a->ld_residual = e->ld_residual;
  if (e->preact) { a->paired = a->paired && pairs(e->preact, e->ld_preact, v.N, v.osize); ld->c = std::max(ld->c, e->ld_preact); }
  if (e->residual) { a->paired = a->paired && pairs(e->residual, e->ld_residual, v.N, v.osize); ld->c = std::max(ld->c, e->ld_residual); }
}

}  // namespace

// ------------------------------------------------------------------------------------ product with epilogue
extern "C" size_t gensor_gemm_fused_workspace_bytes(const gensor_problem* p) {
  size_t bytes = 0;
  guarded([&]() -> gensor_status {
    bytes = [&]() -> size_t {
  GemmView v;
  if (!p || p->op != GENSOR_OP_GEMM || gemm_view(p, &v) != GENSOR_OK || (v.asrc == A_MC && v.bsrc == B_KC)) return 0;
  const LeadingDims ld = {v.asrc == A_KC ? v.K : v.M, v.bsrc == B_KC ? v.K : v.N, v.N};
  size_t most = 0;
  for (int vec = 0; vec < 2; ++vec) {
    FusedChoice c;
    if (choose(v, FUSED_LINEAR, vec != 0, ld, SIZE_MAX, &c) == GENSOR_OK) most = std::max(most, c.bytes);
  }
  return most;
    }();
    return GENSOR_OK;
  });
  return bytes;
}

extern "C" gensor_status gensor_gemm_fused(const gensor_problem* p, const gensor_epilogue* e, float alpha, const void* A, int64_t lda,
                                           const void* B, int64_t ldb, void* C, int64_t ldc, void* workspace, size_t workspace_bytes,
                                           void* hip_stream) {
  return guarded([&]() -> gensor_status {
  if (!p || !A || !B || !C || p->op != GENSOR_OP_GEMM) return GENSOR_ERR_INVALID_ARG;
  GemmView v;
  gensor_status st = gemm_view(p, &v);
  if (st != GENSOR_OK) return st;
  if (lda < (v.asrc == A_KC ? v.K : v.M) || ldb < (v.bsrc == B_KC ? v.K : v.N) || ldc < v.N) return GENSOR_ERR_INVALID_ARG;
  st = check_epilogue(e, v, C);
  if (st != GENSOR_OK) return st;
  if ((v.asrc == A_MC && v.bsrc == B_KC) || !extents_fit(v)) return GENSOR_ERR_UNSUPPORTED;
  FusedArgs a = product_args(v, A, lda, B, ldb, C, ldc, alpha);
  LeadingDims ld = {lda, ldb, ldc};
  set_epilogue(&a, e, v, &ld);
  FusedChoice c;
  st = choose(v, FUSED_LINEAR, vector_ok(v, A, lda, 0, B, ldb, 0), ld, usable_room(workspace, workspace_bytes), &c);
  if (st == GENSOR_ERR_UNSUPPORTED && v.M >= 1 << 20) {
    // More tiles than a launch can have, whichever is taken: the rows in two halves (or rows too far apart, which the first half says, too)
    gensor_problem half = *p;
    half.M = (v.M / 2 + 255) / 256 * 256;
    st = gensor_gemm_fused(&half, e, alpha, A, lda, B, ldb, C, ldc, workspace, workspace_bytes, hip_stream);
    if (st != GENSOR_OK) return st;
    gensor_epilogue rest = e ? *e : gensor_epilogue{};
    if (rest.preact) rest.preact = (char*)rest.preact + half.M * rest.ld_preact * v.osize;
    if (rest.residual) rest.residual = (const char*)rest.residual + half.M * rest.ld_residual * v.osize;
    const char* A2 = (const char*)A + half.M * (v.asrc == A_KC ? lda : 1) * v.esize;
    char* C2 = (char*)C + half.M * ldc * v.osize;
    half.M = v.M - half.M;
    return gensor_gemm_fused(&half, e ? &rest : nullptr, alpha, A2, lda, B, ldb, C2, ldc, workspace, workspace_bytes, hip_stream);
  }
  if (st != GENSOR_OK) return st;
  // Panels of two tile rows: what is read and kept beside C lies closer together.  Two and four, us: 8192 x 3072 x 768 with Z kept 57.4 and 59.0,
  // the gradient through gelu with the bias's 78.6 and 83.0; 16384 x 3072 x 768 102.9 and 102.6, 4096 x 4096 x 1024 38.1 and 37.3, 8192 x 768 x
  // 3072 43.2 both.  (The logits, whose C is not stored, 577 and 566.)
  return run_linear(a, v, c, workspace, (hipStream_t)hip_stream, 2);
  });
}

// ------------------------------------------------------------------------------------ products grouped by expert
namespace {
// p: batch = groups, M = the rows of all groups (0: none), C = A[rows of g] * B[g]
gensor_status grouped_view(const gensor_problem* p, GemmView* v) {
  if (!p || p->op != GENSOR_OP_BMM || p->transA != 0 || p->batch <= 0 || p->M < 0) return GENSOR_ERR_INVALID_ARG;
  gensor_problem q = *p;
  if (q.M == 0) q.M = 1;
  const gensor_status st = gemm_view(&q, v);
  return st == GENSOR_OK && !extents_fit(*v) ? GENSOR_ERR_UNSUPPORTED : st;
}
}  // namespace

extern "C" gensor_status gensor_grouped_gemm(const gensor_problem* p, const int32_t* offsets, const gensor_epilogue* e, float alpha,
                                             const void* A, int64_t lda, const void* B, int64_t ldb, int64_t strideB, void* C, int64_t ldc,
                                             void* hip_stream) {
  return guarded([&]() -> gensor_status {
  GemmView v;
  gensor_status st = grouped_view(p, &v);
  if (st != GENSOR_OK) return st;
  const int64_t rows = p->M, groups = v.batch;
  if (!offsets || !A || !B || !C || !aligned(offsets, 4)) return GENSOR_ERR_INVALID_ARG;
  if (lda < v.K || ldb < (v.bsrc == B_KC ? v.K : v.N) || ldc < v.N || strideB < 0) return GENSOR_ERR_INVALID_ARG;
  st = check_epilogue(e, v, C);
  if (st != GENSOR_OK) return st;
  if (rows == 0) return GENSOR_OK;
  GemmView all = v, each = v;              // one output of all rows; what a group is on average, for the choice of the tile
  all.batch = 1;
  each.M = (rows + groups - 1) / groups;
  FusedArgs a = product_args(all, A, lda, B, ldb, C, ldc, alpha);
  LeadingDims ld = {lda, ldb, ldc};
  set_epilogue(&a, e, v, &ld);
  a.strideB = strideB;
  a.offsets = offsets;
  a.groups = (int32_t)groups;
  a.rows = (int32_t)rows;
  FusedChoice c;
  st = choose(each, FUSED_ROWS, vector_ok(v, A, lda, 0, B, ldb, strideB), ld, 0, &c);
  if (st != GENSOR_OK) return st;
  // Rows of C that do not start on cache lines: the tiles at any alignment, whose own rows are not whole vectors either, leave write-through
  // earlier.  Through and back, us: 8 groups, 8355 x 502 x 120 f16 (8 MB) 9.4 and 8.7, 13345 x 1100 x 264 (28 MB) 26.6 and 24.1, with fp32
  // output 7149 rows (30 MB) 21.3 and 20.5; but 4 MB 7.2 both, fp32 output of 8 MB 10.4 and 10.9.  Aligned: 16 groups, 8192 x 1000 x 256 (16 MB) 19.5 and
  // 20.8, 8192 x 1400 x 352 (22 MB) 18.0 and 19.8.
  if (!c.f->d.vec && (ldc * v.osize) % 128 != 0) a.through = rows * v.N * v.osize <= (v.osize == 2 ? 4ll : 16ll) * 1024 * 1024;
  tiles_of(&a, v, c, rows, v.N);
  // whole tiles of the rows, and one more of each group that can have rows; in several launches where one cannot have them
  const int64_t tile_rows = rows / c.f->d.bm + std::min(groups, rows);
  if (tile_rows * a.tiles_n > INT32_MAX) return GENSOR_ERR_UNSUPPORTED;
  a.panel = 4;
  a.batch = 1;
  const int64_t most = std::max<int64_t>(1, UINT32_MAX / c.f->d.threads / a.tiles_n);
  for (int64_t at = 0; at < tile_rows; at += most) {
    a.tile_first = (int32_t)(at * a.tiles_n);
    a.tiles_m = (int32_t)std::min(most, tile_rows - at);
    if (c.f->launch[FUSED_ROWS](a, (hipStream_t)hip_stream) != hipSuccess) return GENSOR_ERR_DEVICE;
  }
  return GENSOR_OK;
  });
}

extern "C" gensor_status gensor_grouped_wgrad(const gensor_problem* p, const int32_t* offsets, const void* A, int64_t lda, const void* dY,
                                              int64_t lddy, void* dW, int64_t lddw, int64_t stride_dw, void* hip_stream) {
  return guarded([&]() -> gensor_status {
  GemmView f;
  gensor_status st = grouped_view(p, &f);
  if (st != GENSOR_OK) return st;
  const int64_t rows = p->M, groups = f.batch;
  if (!offsets || !dW || !aligned(offsets, 4) || (rows > 0 && (!A || !dY))) return GENSOR_ERR_INVALID_ARG;
  // dW[g] = A_g^T dY_g as [K][N], or dY_g^T A_g as [N][K]
  const bool swapped = f.bsrc == B_KC;
  const int64_t m = swapped ? f.N : f.K, n = swapped ? f.K : f.N;
  if (lda < f.K || lddy < f.N || lddw < n || stride_dw < 0) return GENSOR_ERR_INVALID_ARG;
  if (groups > 1 && stride_dw < m * lddw - (lddw - n)) return GENSOR_ERR_INVALID_ARG;      // outputs must not overlap
  const void* L = swapped ? dY : A;
  const void* R = swapped ? A : dY;
  const int64_t ldl = swapped ? lddy : lda, ldr = swapped ? lda : lddy;
  const GemmView v = product_view(f.in_dtype, f.out_dtype, m, n, std::max<int64_t>(1, (rows + groups - 1) / groups), A_MC, B_NC, groups);
  FusedArgs a = product_args(v, L, ldl, R, ldr, dW, lddw, 1.f);
  a.strideC = stride_dw;
  a.paired = pairs(dW, lddw, n, v.osize) && stride_dw % 2 == 0;
  a.offsets = offsets;
  a.groups = (int32_t)groups;
  a.rows = (int32_t)rows;
  const LeadingDims ld = {ldl, ldr, lddw};
  FusedChoice c;
  st = choose(v, FUSED_DEPTH, vector_ok(v, L, ldl, 0, R, ldr, 0), ld, 0, &c);
  if (st == GENSOR_ERR_UNSUPPORTED && groups >= 1 << 10) {
    // more tiles than a launch can have: the groups in two halves (their rows stay where they are)
    gensor_problem half = *p;
    half.batch = groups / 2;
    st = gensor_grouped_wgrad(&half, offsets, A, lda, dY, lddy, dW, lddw, stride_dw, hip_stream);
    if (st != GENSOR_OK) return st;
    char* dW2 = (char*)dW + half.batch * stride_dw * v.osize;
    const int32_t* offsets2 = offsets + half.batch;
    half.batch = groups - half.batch;
    return gensor_grouped_wgrad(&half, offsets2, A, lda, dY, lddy, dW2, lddw, stride_dw, hip_stream);
  }
  if (st != GENSOR_OK) return st;
  tiles_of(&a, v, c, m, n);
  return launched(c.f->launch[FUSED_DEPTH](a, (hipStream_t)hip_stream));
  });
}

// ------------------------------------------------------------------------------------ column sums
// db[g][n] = sum of dY[r][n] over the rows of g, fp32 sums.  Bound by reading dY once.  A workgroup takes 64 vectors' columns and one of `parts`
// equal shares of a group's rows; its eight waves take turns at the rows, eight rows requested together, and add up in LDS.  The shares'
// sums go to the workspace and a second launch adds them in order, so the result does not depend on when a share finished.  8192 x 3072 bf16: 9.6 to 17 us
// (3 to 5.2 TB/s) and 3 to 5 for the shares; with four waves, four rows each and 171 shares 18 and 14.
namespace gensor {

template <typename T, typename OutT, bool VEC>
__global__ __launch_bounds__(512) void column_sums_kernel(const char* Y, int64_t ld, int rows, int N, const int32_t* offsets, int groups, int parts,
                                                          float* partial, void* out) {
  constexpr int ES = ElemSize<T>::value, EPC = 16 / ES, UNROLL = VEC ? 8 : 4, WAVES = 8;
  __shared__ float sums[WAVES][64 * EPC];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = blockIdx.z, part = blockIdx.y;
  int first = 0, count = rows;
  if (offsets) {
    first = min(max(offsets[g], 0), rows);
    count = min(max(offsets[g + 1], first), rows) - first;
  }
  const int r0 = first + (int)((int64_t)part * count / parts), r1 = first + (int)((int64_t)(part + 1) * count / parts);
  const int col0 = blockIdx.x * 64 * EPC;
  float acc[EPC];
#pragma unroll
  for (int e = 0; e < EPC; ++e) acc[e] = 0.f;
  // element e of a lane is column col0 + EPC * lane + e (vectors) or col0 + lane + 64 * e
  const int mine = VEC ? col0 + lane * EPC : col0 + lane;
  for (int r = r0 + wave; r < r1; r += WAVES * UNROLL) {
    if constexpr (VEC) {
      u32x4 v[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        v[u] = u32x4{0u, 0u, 0u, 0u};
        if (r + WAVES * u < r1 && mine < N) v[u] = *(const u32x4*)(Y + ((int64_t)(r + WAVES * u) * ld + mine) * ES);
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u)
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          if constexpr (ES == 4) acc[e] += as_f32(v[u][e]);
          else acc[e] += from_pair<T>(v[u][e / 2], e & 1);
        }
    } else {
#pragma unroll
      for (int u = 0; u < UNROLL; ++u)
#pragma unroll
        for (int e = 0; e < EPC; ++e)
          if (r + WAVES * u < r1 && mine + 64 * e < N) acc[e] += to_float<T>(Y, (int64_t)(r + WAVES * u) * ld + mine + 64 * e);
    }
  }
#pragma unroll
  for (int e = 0; e < EPC; ++e) sums[wave][VEC ? lane * EPC + e : lane + 64 * e] = acc[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * EPC; i += 512) {
    const int col = col0 + i;
    if (col >= N) continue;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += sums[w][i];
    if (parts == 1) store_out<OutT>(out, (int64_t)g * N + col, s);
    else partial[((int64_t)g * parts + part) * N + col] = s;
  }
}

template <typename OutT>
__global__ __launch_bounds__(1024) void column_parts_kernel(const float* partial, int parts, int N, void* out) {
  constexpr int WAVES = 16, UNROLL = 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
  __shared__ float sums[WAVES][64];
  float s = 0.f;
  for (int p = wave; p < parts; p += WAVES * UNROLL) {
    float v[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) v[u] = col < N && p + WAVES * u < parts ? partial[((int64_t)blockIdx.y * parts + p + WAVES * u) * N + col] : 0.f;
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) s += v[u];
  }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || col >= N) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) s += sums[w][lane];
  store_out<OutT>(out, (int64_t)blockIdx.y * N + col, s);
}

}  // namespace gensor

namespace {
// Shares of a group's rows: enough that the launch has about four workgroups a compute unit, none of fewer than 64 rows on average.
int64_t column_parts(int64_t groups, int64_t rows, int64_t N, int esize) {
  const int64_t blocks = (N + 64 * (16 / esize) - 1) / (64 * (16 / esize)) * groups;
  const int64_t want = (4 * 256 + blocks - 1) / blocks, most = std::max<int64_t>(1, rows / groups / 64);
  return std::min<int64_t>(std::min(want, most), 1024);
}

template <typename T, typename OutT>
gensor_status launch_columns(const void* dY, int64_t ld, int64_t rows, int64_t N, const int32_t* offsets, int64_t groups, int64_t parts, bool vec,
                             void* out, float* partial, hipStream_t st) {
  const int64_t per = 64 * (16 / ElemSize<T>::value);
  const dim3 grid((unsigned)((N + per - 1) / per), (unsigned)parts, (unsigned)groups);
  if (vec)
    hipLaunchKernelGGL((column_sums_kernel<T, OutT, true>), grid, dim3(512), 0, st, (const char*)dY, ld, (int)rows, (int)N, offsets, (int)groups, (int)parts, partial, out);
  else
    hipLaunchKernelGGL((column_sums_kernel<T, OutT, false>), grid, dim3(512), 0, st, (const char*)dY, ld, (int)rows, (int)N, offsets, (int)groups, (int)parts, partial, out);
  if (hipGetLastError() != hipSuccess) return GENSOR_ERR_DEVICE;
  if (parts == 1) return GENSOR_OK;
  hipLaunchKernelGGL((column_parts_kernel<OutT>), dim3((unsigned)((N + 63) / 64), (unsigned)groups), dim3(1024), 0, st, partial, (int)parts, (int)N, out);
  return launched(hipGetLastError());
}
}  // namespace

extern "C" size_t gensor_bias_grad_workspace_bytes(gensor_dtype in_dtype, int64_t groups, int64_t rows, int64_t N) {
  if (!valid_dtype(in_dtype) || groups <= 0 || rows < 0 || N <= 0) return 0;
  const int64_t parts = column_parts(groups, rows, N, size_of(in_dtype));
  return parts > 1 ? (size_t)(groups * parts * N * 4) : 0;
}

extern "C" gensor_status gensor_bias_grad(gensor_dtype in_dtype, gensor_dtype out_dtype, int64_t groups, int64_t rows, int64_t N,
                                          const void* dY, int64_t ld, const int32_t* offsets, void* db, void* workspace, size_t workspace_bytes,
                                          void* hip_stream) {
  if (!valid_dtype(in_dtype) || !valid_dtype(out_dtype)) return GENSOR_ERR_INVALID_ARG;
  if (groups <= 0 || rows < 0 || N <= 0 || ld < N || !db || (rows > 0 && !dY)) return GENSOR_ERR_INVALID_ARG;
  if ((!offsets && groups != 1) || (offsets && !aligned(offsets, 4))) return GENSOR_ERR_INVALID_ARG;
  if (out_dtype != GENSOR_F32 && out_dtype != in_dtype) return GENSOR_ERR_UNSUPPORTED;
  if (rows > INT32_MAX - 64 || N > INT32_MAX - 4096 || groups > 65535) return GENSOR_ERR_UNSUPPORTED;
  const int es = size_of(in_dtype);
  int64_t parts = column_parts(groups, rows, N, es);
  // (shares of fewer rows than the workspace has room for: no error, only fewer of them)
  const size_t room = workspace && aligned(workspace, 4) ? workspace_bytes : 0;
  if (parts > 1 && (size_t)(groups * parts * N * 4) > room) parts = std::max<int64_t>(1, (int64_t)(room / (size_t)(groups * N * 4)));
  const bool vec = aligned(dY, 16) && ld % (16 / es) == 0 && N % (16 / es) == 0;
  hipStream_t st = (hipStream_t)hip_stream;
  float* partial = (float*)workspace;
  if (in_dtype == GENSOR_F32) return launch_columns<f32_t, f32_t>(dY, ld, rows, N, offsets, groups, parts, vec, db, partial, st);
  if (in_dtype == GENSOR_F16)
    return out_dtype == GENSOR_F32 ? launch_columns<f16_t, f32_t>(dY, ld, rows, N, offsets, groups, parts, vec, db, partial, st)
                                   : launch_columns<f16_t, f16_t>(dY, ld, rows, N, offsets, groups, parts, vec, db, partial, st);
  return out_dtype == GENSOR_F32 ? launch_columns<bf16_t, f32_t>(dY, ld, rows, N, offsets, groups, parts, vec, db, partial, st)
                                 : launch_columns<bf16_t, bf16_t>(dY, ld, rows, N, offsets, groups, parts, vec, db, partial, st);
}

// ------------------------------------------------------------------------------------ cross entropy of a projection
namespace gensor {

// The slabs' maxima and sums of a token joined.  A workgroup takes `per` tokens (a power of two); the threads of a token take turns at
// the slabs, several requested together, and are joined in LDS.  keep_max: the slabs of further pieces follow, so what there is so far is left
// there (it may be the first of the slabs) in place of results.
__global__ __launch_bounds__(1024) void xent_join_kernel(const float* part_max, const float* part_sum, int slabs, int tokens, int per, float* keep_max, float* keep_sum,
                                                         const int64_t* targets, int64_t ignore, int vocab, const float* at_target, float* loss, float* lse) {
  constexpr int UNROLL = 4;
  __shared__ float tops[1024], sums[1024];
  const int i = threadIdx.x, lanes = 1024 / per, lane = i / per;
  const int t = blockIdx.x * per + i % per;
  float top = -INFINITY, sum = 0.f;
  for (int s = lane; s < slabs; s += UNROLL * lanes) {
    float m[UNROLL], x[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const bool there = t < tokens && s + u * lanes < slabs;
      const int64_t at = (int64_t)(s + u * lanes) * tokens + t;
      m[u] = there ? part_max[at] : -INFINITY;
      x[u] = there ? part_sum[at] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) join_sums(top, sum, m[u], x[u]);
  }
  tops[i] = top;
  sums[i] = sum;
  for (int half = lanes / 2; half >= 1; half /= 2) {
    __syncthreads();
    if (lane < half) {
      join_sums(top, sum, tops[i + half * per], sums[i + half * per]);
      tops[i] = top;
      sums[i] = sum;
    }
  }
  if (lane != 0 || t >= tokens) return;
  if (keep_max) {
    keep_max[t] = top;
    keep_sum[t] = sum;
    return;
  }
  const float ref = lse_reference(top), rest = logf(sum);
  if (lse) lse[t] = ref + rest;
  if (loss) {
    const int64_t target = targets[t];
    // (the maximum's part first: a token whose target is the maximum loses log(1 + the others), not a difference of large numbers)
    loss[t] = target == ignore ? 0.f : target >= 0 && target < vocab ? (ref - at_target[t]) + rest : NAN;
  }
}

// G is rounded to the type, and most of it is -dloss at the targets: where all tokens have the same dloss (1 / 401 is 0.26 % off in bf16, 0.035 in f16) that
// would be one common factor of both gradients.  So G is scaled to make the largest dloss of the tokens that count 2^15, which both types
// have and which fills f16's range (gradients of a mean are below its normal one); the products undo it in fp32.  (The other tokens' G is zero,
// whatever stands there: 1e8 at padding would leave the rest f16's last bits.)  scale[0] = the factor, scale[1] its inverse.
__global__ __launch_bounds__(1024) void xent_scale_kernel(const float* dloss, const int64_t* targets, int64_t ignore, int vocab, int tokens, float* scale) {
  constexpr int UNROLL = 8;
  __shared__ float tops[16];
  float top = 0.f;
  for (int first = threadIdx.x; first < tokens; first += UNROLL * 1024) {
    float x[UNROLL];
    int64_t target[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const bool there = first + u * 1024 < tokens;
      x[u] = there ? fabsf(dloss[first + u * 1024]) : 0.f;
      target[u] = there ? targets[first + u * 1024] : ignore;
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
      if (x[u] < INFINITY && target[u] != ignore && target[u] >= 0 && target[u] < vocab) top = fmaxf(top, x[u]);
  }
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < 16; ++w) top = fmaxf(top, tops[w]);
  const float f = top > 0.f ? fminf(fmaxf(32768.f / top, 0x1p-100f), 0x1p100f) : 1.f;
  scale[0] = f;
  scale[1] = 1.f / f;
}

// rows of D elements copied to rows of D elements, `padded` of them, those behind `rows` zero
template <int ES>
__global__ __launch_bounds__(256) void xent_pad_kernel(const char* X, int64_t ld, int rows, int padded, int D, char* out) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)padded * D; i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i / D), c = (int)(i - (int64_t)r * D);
    if constexpr (ES == 4) ((uint32_t*)out)[i] = r < rows ? ((const uint32_t*)X)[(int64_t)r * ld + c] : 0u;
    else ((uint16_t*)out)[i] = r < rows ? ((const uint16_t*)X)[(int64_t)r * ld + c] : (uint16_t)0;
  }
}

}  // namespace gensor

namespace {

gensor_status check_xent(gensor_dtype dtype, int64_t T, int64_t V, int64_t D) {
  if (!valid_dtype(dtype) || T <= 0 || V <= 0 || D <= 0) return GENSOR_ERR_INVALID_ARG;
  if (T > INT32_MAX / 8 || V > INT32_MAX / 8 || D > INT32_MAX / 8) return GENSOR_ERR_UNSUPPORTED;
  return GENSOR_OK;
}

size_t round_up(size_t n, size_t to) { return (n + to - 1) / to * to; }

size_t lse_bytes(int64_t T, int64_t V, int wm) { return round_up((size_t)((V + wm - 1) / wm * T * 4), 256); }

// The gradient's workspace: [scales 256][padded X][fp32 sums of dX][partial tiles][pieces of G].  G of a piece has n rows (vocabulary
// entries) of `pitch` tokens.
struct XentPlan {
  int64_t pitch, piece, pieces;
  bool pad;
  size_t pad_bytes, sum_bytes, part_bytes, piece_bytes, total;
};

// A piece's G at most: larger pieces fill the chip in more whole rounds and split dX's sum less often (50257 entries, 4096 tokens, 768 wide, bf16: in a
// workspace of 64 MiB 1721 us, 128 1259, 192 1082, 306, as asked for with pieces of 256 at most, 866), but the logits of a batch are not to be kept.
const size_t kPieceBytes = (size_t)256 << 20;
const size_t kPartBytes = (size_t)64 << 20;

// The gradient of 4096 tokens over 50257 entries of width 768 in bf16, 866 us (1.10 PFLOP/s of the six 2TVD): logits again 337 to 361, dW 271 to 286, dX 241 to
// 260 and its partial tiles' sums 39, the scale 5.
// The cheapest whole or split tile's price, not remembered.
double best_price(const GemmView& v, int kind, bool vec, size_t room) {
  const LeadingDims ld = {v.asrc == A_KC ? v.K : v.M, v.bsrc == B_KC ? v.K : v.N, v.N};
  double best = 1e30;
  for (int i = 0; i < g_num_fused; ++i) {
    const FusedDesc& f = g_fused[i];
    if (!f.launch[kind] || f.d.vec != (vec ? 1 : 0) || !instance_serves(f.d, v) || !offsets_fit(f.d, v, ld) || !tiles_fit(f.d, v, kind)) continue;
    for (int split : kSplits) {
      if (split > 1 && (kind != FUSED_LINEAR || (v.K + f.d.bk - 1) / f.d.bk < split)) break;
      const double us = tile_price(f, v, kind, split);
      if (us > 0 && us < best && split_plan(f.d, v, split, 0).bytes <= room) best = us;
    }
  }
  return best;
}

GemmView prob_view(int dtype, int64_t rows, int64_t T, int64_t D) { return product_view(dtype, dtype, rows, T, D, A_KC, B_KC); }
GemmView dw_view(int dtype, int64_t rows, int64_t pitch, int64_t D) { return product_view(dtype, dtype, rows, D, pitch, A_KC, B_NC); }
GemmView dx_view(int dtype, int64_t rows, int64_t pitch, int64_t D, bool last) {
  return product_view(dtype, last ? dtype : (int)GENSOR_F32, pitch, D, rows, A_MC, B_NC);
}

std::map<std::array<int64_t, 6>, int64_t> g_piece_sizes;         // guarded by g_choice_mutex

// Entries of a piece where V of them do not fit one of `most`: all pieces but the last have as many.  A piece's products each end in a partly
// filled round of tiles, so the sizes in steps of a tile are priced: 50257 entries for 4096 tokens in pieces of 12800 (four rounds
// of 256x256 tiles, the last almost empty) 1051 us, of 25344 956.
int64_t piece_size(int dtype, int64_t T, int64_t V, int64_t D, int64_t pitch, int64_t most) {
  const bool vec = D % (16 / size_of(dtype)) == 0;
  auto price = [&](int64_t rows, bool last) {
    return best_price(prob_view(dtype, rows, T, D), FUSED_PROB, vec, 0) + best_price(dw_view(dtype, rows, pitch, D), FUSED_LINEAR, vec, kPartBytes) +
           best_price(dx_view(dtype, rows, pitch, D, last), FUSED_LINEAR, vec, kPartBytes);
  };
  const int64_t least = (V + most - 1) / most;             // pieces
  int64_t best = most, step = 256;
  while (most / step > 64) step *= 2;                      // at most 64 sizes of each count are priced
  double best_us = 1e30;
  for (int64_t n = least; n <= least + 1; ++n)
    for (int64_t size = (V / n + 255) / 256 * 256; size <= most && (n - 1) * size < V; size += step) {
      const int64_t last = V - (n - 1) * size;
      if (last > most) continue;
      const double us = (double)(n - 1) * price(size, false) + price(last, true);
      if (us < best_us) { best_us = us; best = size; }
    }
  return best;
}

bool plan_xent(int dtype, int64_t T, int64_t V, int64_t D, size_t room, XentPlan* pl) {
  const int es = size_of(dtype), epc = 16 / es;
  pl->pitch = (T + epc - 1) / epc * epc;
  pl->pad = pl->pitch != T;
  pl->pad_bytes = pl->pad ? round_up((size_t)(pl->pitch * D * es), 256) : 0;
  const size_t row = (size_t)(pl->pitch * es);
  int64_t most = std::max<int64_t>(256, (int64_t)(kPieceBytes / row) / 256 * 256);
  auto layout = [&]() {
    pl->piece = V;
    if (V > most) {
      const std::array<int64_t, 6> key = {dtype, T, V, D, pl->pitch, most};
      std::lock_guard<std::mutex> lock(g_choice_mutex);
      auto it = g_piece_sizes.find(key);
      if (it == g_piece_sizes.end()) {
        if (g_piece_sizes.size() >= kChoiceLimit) g_piece_sizes.clear();
        it = g_piece_sizes.emplace(key, piece_size(dtype, T, V, D, pl->pitch, most)).first;
      }
      pl->piece = it->second;
    }
    pl->pieces = (V + pl->piece - 1) / pl->piece;
    // (a last piece that is larger than the others: what it has more would be a small piece of its own)
    while (pl->pieces > 1 && V - (pl->pieces - 2) * pl->piece <= most) --pl->pieces;
    const int64_t largest = std::max(pl->piece, V - (pl->pieces - 1) * pl->piece);
    pl->sum_bytes = pl->pieces > 1 && dtype != GENSOR_F32 ? round_up((size_t)(T * D * 4), 256) : 0;
    pl->piece_bytes = round_up((size_t)largest * row, 256);
    // the room the products' partial tiles would like, within a limit
    size_t parts = 0;
    for (int64_t rows : {pl->piece, V - (pl->pieces - 1) * pl->piece}) {
      const bool last = rows != pl->piece || pl->pieces == 1;
      const GemmView dw = dw_view(dtype, rows, pl->pitch, D), dx = dx_view(dtype, rows, pl->pitch, D, last);
      for (const GemmView* v : {&dw, &dx})
        for (int vec = 0; vec < 2; ++vec) {
          FusedChoice c;
          const LeadingDims ld = {pl->pitch, D, D};
          if (choose(*v, FUSED_LINEAR, vec != 0, ld, kPartBytes, &c) == GENSOR_OK) parts = std::max(parts, c.bytes);
        }
    }
    pl->part_bytes = round_up(parts, 256);
    pl->total = 256 + pl->pad_bytes + pl->sum_bytes + pl->part_bytes + pl->piece_bytes;
  };
  layout();
  while (pl->total > room && most > 256) {                 // less room: smaller pieces
    most = std::max<int64_t>(256, most / 2 / 256 * 256);
    layout();
  }
  if (pl->total > room) {                                  // and no partial tiles
    pl->total -= pl->part_bytes;
    pl->part_bytes = 0;
  }
  return pl->total <= room;
}

gensor_status choose_logits(int dtype, int kind, int64_t rows, int64_t T, int64_t D, const void* W, int64_t ldw, const void* X, int64_t ldx, int64_t ldc,
                            GemmView* v, FusedChoice* c) {
  *v = prob_view(dtype, rows, T, D);
  const LeadingDims ld = {ldw, ldx, ldc};
  return choose(*v, kind, vector_ok(*v, W, ldw, 0, X, ldx, 0), ld, 0, c);
}

}  // namespace

extern "C" size_t gensor_xent_workspace_bytes(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, int32_t backward) {
  size_t bytes = 0;
  guarded([&]() -> gensor_status {
    bytes = [&]() -> size_t {
  if (check_xent(dtype, T, V, D) != GENSOR_OK) return 0;
  if (backward) {
    XentPlan pl;
    plan_xent(dtype, T, V, D, SIZE_MAX, &pl);
    return pl.total;
  }
  // whichever tile the operands' alignment leads to, and, for rows so far apart that a smaller tile serves them, a piece of any tile's
  const GemmView v = product_view(dtype, dtype, V, T, D, A_KC, B_KC);
  size_t most = 0;
  for (int vec = 0; vec < 2; ++vec) {
    FusedChoice c;
    const LeadingDims ld = {D, D, 0};
    if (choose(v, FUSED_LSE, vec != 0, ld, 0, &c) == GENSOR_OK) most = std::max(most, lse_bytes(T, V, c.f->d.wm));
  }
  for (int i = 0; i < g_num_fused; ++i) {
    const InstanceDesc& d = g_fused[i].d;
    if (g_fused[i].launch[FUSED_LSE] && instance_serves(d, v)) most = std::max(most, lse_bytes(T, std::min<int64_t>(V, d.bm + d.wm), d.wm));
  }
  return round_up((size_t)T * 4, 256) + 2 * most;
    }();
    return GENSOR_OK;
  });
  return bytes;
}

extern "C" gensor_status gensor_xent_forward(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx, const void* W, int64_t ldw,
                                             const int64_t* targets, int64_t ignore_index, float* loss, float* lse, void* workspace,
                                             size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> gensor_status {
  gensor_status st = check_xent(dtype, T, V, D);
  if (st != GENSOR_OK) return st;
  if (!X || !W || (!loss && !lse) || (loss && !targets) || ldx < D || ldw < D || (targets && !aligned(targets, 8))) return GENSOR_ERR_INVALID_ARG;
  GemmView v;
  FusedChoice c;
  st = choose_logits(dtype, FUSED_LSE, V, T, D, W, ldw, X, ldx, 0, &v, &c);
  if (st == GENSOR_ERR_UNSUPPORTED && T >= 1 << 20) {
    // more tiles than a launch can have: the tokens in two halves
    const int64_t half = (T / 2 + 255) / 256 * 256;
    st = gensor_xent_forward(dtype, half, V, D, X, ldx, W, ldw, targets, ignore_index, loss, lse, workspace, workspace_bytes, hip_stream);
    if (st != GENSOR_OK) return st;
    return gensor_xent_forward(dtype, T - half, V, D, (const char*)X + half * ldx * size_of(dtype), ldx, W, ldw, targets ? targets + half : nullptr, ignore_index,
                               loss ? loss + half : nullptr, lse ? lse + half : nullptr, workspace, workspace_bytes, hip_stream);
  }
  if (st != GENSOR_OK) return st;
  const InstanceDesc& d = c.f->d;
  const size_t room = usable_room(workspace, workspace_bytes), head = round_up((size_t)T * 4, 256);
  // Room for fewer slabs than the vocabulary has (rows that are far apart lead to smaller tiles, of more slabs, than the room was asked for): pieces of
  // as many whole tiles' rows as fit, evened out.  Slab 0 is what the pieces in front have been joined to.
  int64_t piece = V, pieces = 1;
  size_t each = lse_bytes(T, V, d.wm);
  if (room < head + 2 * each) {
    each = room > head ? (room - head) / 2 / 256 * 256 : 0;
    const int64_t most = ((int64_t)(each / ((size_t)T * 4)) - 1) * d.wm / d.bm * d.bm;
    if (most <= 0) return GENSOR_ERR_WORKSPACE;
    pieces = (V + most - 1) / most;
    piece = ((V + pieces - 1) / pieces + d.bm - 1) / d.bm * d.bm;
    pieces = (V + piece - 1) / piece;
  }
  hipStream_t s = (hipStream_t)hip_stream;
  float* at_target = (float*)workspace;
  float* tops = (float*)((char*)workspace + head);
  float* sums = (float*)((char*)workspace + head + each);
  int per = 1;
  while (per < 32 && per < T) per *= 2;          // whole lines (of 8192 tokens: 3 us of 612 less than with 16, 15 less than with 8)
  while (!launch_fits((double)((T + per - 1) / per), 1024)) per *= 2;
  for (int64_t i = 0; i < pieces; ++i) {
    const bool first = i == 0, last = i + 1 == pieces;
    const int64_t entry = i * piece, rows = last ? V - entry : piece, kept = pieces > 1 ? T : 0;
    const GemmView q = prob_view(dtype, rows, T, D);
    FusedArgs a = product_args(q, (const char*)W + entry * ldw * size_of(dtype), ldw, X, ldx, nullptr, 0, 1.f);
    a.targets = loss ? targets : nullptr;
    a.ignore = ignore_index;
    a.tokens = (int32_t)T;
    a.row_first = (int32_t)entry;
    a.vocab = (int32_t)V;
    a.at_target = at_target;
    a.part_max = tops + kept;
    a.part_sum = sums + kept;
    tiles_of(&a, q, c, rows, T);
    if (c.f->launch[FUSED_LSE](a, s) != hipSuccess) return GENSOR_ERR_DEVICE;
    const int64_t from = first ? kept : 0;
    const int slabs = (int)((rows + d.wm - 1) / d.wm) + (first ? 0 : 1);
    hipLaunchKernelGGL(xent_join_kernel, dim3((unsigned)((T + per - 1) / per)), dim3(1024), 0, s, tops + from, sums + from, slabs, (int)T, per,
                       last ? nullptr : tops, last ? nullptr : sums, targets, ignore_index, (int)V, at_target, loss, lse);
    if (hipGetLastError() != hipSuccess) return GENSOR_ERR_DEVICE;
  }
  return GENSOR_OK;
  });
}

extern "C" gensor_status gensor_xent_backward(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx, const void* W, int64_t ldw,
                                              const int64_t* targets, int64_t ignore_index, const float* lse, const float* dloss, void* dX,
                                              int64_t lddx, void* dW, int64_t lddw, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> gensor_status {
  gensor_status st = check_xent(dtype, T, V, D);
  if (st != GENSOR_OK) return st;
  if (!X || !W || !targets || !lse || !dloss || (!dX && !dW) || ldx < D || ldw < D || (dX && lddx < D) || (dW && lddw < D) || !aligned(targets, 8))
    return GENSOR_ERR_INVALID_ARG;
  XentPlan pl;
  if (!plan_xent(dtype, T, V, D, usable_room(workspace, workspace_bytes), &pl)) return GENSOR_ERR_WORKSPACE;
  const int es = size_of(dtype);
  char* at = (char*)workspace;
  float* scales = (float*)at;
  char* padded = at + 256;
  float* sums = (float*)(padded + pl.pad_bytes);
  char* parts = (char*)sums + pl.sum_bytes;
  char* G = parts + pl.part_bytes;
  hipStream_t s = (hipStream_t)hip_stream;
  const bool scaled = dtype != GENSOR_F32;

  // every product's tile is chosen before anything is launched
  struct Piece { int64_t first, rows; GemmView vp, vw, vx; FusedChoice cp, cw, cx; };
  std::vector<Piece> pieces((size_t)pl.pieces);
  const void* Xs = pl.pad ? (const void*)padded : X;
  const int64_t ldxs = pl.pad ? D : ldx;
  for (int64_t i = 0; i < pl.pieces; ++i) {
    Piece& q = pieces[(size_t)i];
    q.first = i * pl.piece;
    q.rows = i + 1 == pl.pieces ? V - q.first : pl.piece;
    const char* Wp = (const char*)W + q.first * ldw * es;
    st = choose_logits(dtype, FUSED_PROB, q.rows, T, D, Wp, ldw, X, ldx, pl.pitch, &q.vp, &q.cp);
    if (st != GENSOR_OK) return st;
    if (dW) {
      q.vw = dw_view(dtype, q.rows, pl.pitch, D);
      const LeadingDims ld = {pl.pitch, ldxs, lddw};
      st = choose(q.vw, FUSED_LINEAR, vector_ok(q.vw, G, pl.pitch, 0, Xs, ldxs, 0), ld, pl.part_bytes, &q.cw);
      if (st != GENSOR_OK) return st;
    }
    if (dX) {
      const bool last = i + 1 == pl.pieces;
      q.vx = dx_view(dtype, q.rows, pl.pitch, D, last);
      const LeadingDims ld = {pl.pitch, ldw, std::max(lddx, D) * (last && dtype != GENSOR_F32 ? 2 : 1)};
      st = choose(q.vx, FUSED_LINEAR, vector_ok(q.vx, G, pl.pitch, 0, Wp, ldw, 0), ld, pl.part_bytes, &q.cx);
      if (st != GENSOR_OK) return st;
    }
  }
  if (scaled) {
    hipLaunchKernelGGL(xent_scale_kernel, dim3(1), dim3(1024), 0, s, dloss, targets, ignore_index, (int)V, (int)T, scales);
    if (hipGetLastError() != hipSuccess) return GENSOR_ERR_DEVICE;
  }
  if (pl.pad && dW) {
    // (a launch has fewer than 2^32 threads along an axis, and the rest is cut off without an error)
    const unsigned blocks = (unsigned)std::min<int64_t>((pl.pitch * D + 255) / 256, 1 << 20);
    if (es == 4) hipLaunchKernelGGL(xent_pad_kernel<4>, dim3(blocks), dim3(256), 0, s, (const char*)X, ldx, (int)T, (int)pl.pitch, (int)D, padded);
    else hipLaunchKernelGGL(xent_pad_kernel<2>, dim3(blocks), dim3(256), 0, s, (const char*)X, ldx, (int)T, (int)pl.pitch, (int)D, padded);
    if (hipGetLastError() != hipSuccess) return GENSOR_ERR_DEVICE;
  }
  for (int64_t i = 0; i < pl.pieces; ++i) {
    Piece& q = pieces[(size_t)i];
    const bool first = i == 0, last = i + 1 == pl.pieces;
    const char* Wp = (const char*)W + q.first * ldw * es;
    {
      FusedArgs a = product_args(q.vp, Wp, ldw, X, ldx, G, pl.pitch, 1.f);
      a.store_n = (int32_t)pl.pitch;
      a.paired = es == 2;
      a.scale = scaled ? scales : nullptr;
      a.targets = targets;
      a.ignore = ignore_index;
      a.lse = lse;
      a.dloss = dloss;
      a.tokens = (int32_t)T;
      a.row_first = (int32_t)q.first;
      a.vocab = (int32_t)V;
      tiles_of(&a, q.vp, q.cp, q.rows, pl.pitch);
      if (q.cp.f->launch[FUSED_PROB](a, s) != hipSuccess) return GENSOR_ERR_DEVICE;
    }
    if (dW) {
      char* dWp = (char*)dW + q.first * lddw * es;
      FusedArgs a = product_args(q.vw, G, pl.pitch, Xs, ldxs, dWp, lddw, 1.f);
      a.paired = pairs(dWp, lddw, D, es);
      a.scale = scaled ? scales + 1 : nullptr;
      st = run_linear(a, q.vw, q.cw, parts, s);
      if (st != GENSOR_OK) return st;
    }
    if (dX) {
      // the pieces' sums: in fp32, in the workspace or, for fp32 gradients, in place; the last piece adds and rounds
      const bool inplace = dtype == GENSOR_F32;
      void* C = last || inplace ? dX : (void*)sums;
      const int64_t ldc = last || inplace ? lddx : D;
      FusedArgs a = product_args(q.vx, G, pl.pitch, Wp, ldw, C, ldc, 1.f);
      a.store_m = (int32_t)T;
      a.scale = scaled ? scales + 1 : nullptr;
      if (!first) {
        a.residual = inplace ? dX : (const void*)sums;
        a.ld_residual = inplace ? lddx : D;
        a.residual_f32 = q.vx.osize == 2;
      }
      a.paired = first && last && pairs(C, ldc, D, q.vx.osize);
      st = run_linear(a, q.vx, q.cx, parts, s);
      if (st != GENSOR_OK) return st;
    }
  }
  return GENSOR_OK;
  });
}
