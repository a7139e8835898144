// C ABI of the gated layers, the scores of a vocabulary and learning from a teacher (gensor_lm.h).  Argument validation, the choice of the
// tiles, the launches and the small kernels between the products.  No device memory is allocated here.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <array>
#include <cmath>
#include <cstring>
#include <map>
#include <mutex>
#include <vector>

#include "../../include/gensor_lm.h"
#include "fused_host.hpp"
#include "lm_registry.hpp"
#include "score_order.hpp"

using namespace gensor;

// ------------------------------------------------------------------------------------ gated layers
namespace {

// The tile that a shape's calls take, remembered: the index in its table, -1 where none serves.
std::mutex g_gated_mutex;
std::map<std::array<int64_t, 12>, int> g_gated_choices;
const size_t kGatedLimit = 4096;

template <typename F>
gensor_status remembered(const std::array<int64_t, 12>& key, int* out, F&& find) {
  std::lock_guard<std::mutex> lock(g_gated_mutex);
  auto it = g_gated_choices.find(key);
  if (it == g_gated_choices.end()) {
    if (g_gated_choices.size() >= kGatedLimit) g_gated_choices.clear();
    it = g_gated_choices.emplace(key, find()).first;
  }
  *out = it->second;
  return *out >= 0 ? GENSOR_OK : GENSOR_ERR_UNSUPPORTED;
}

// The cheapest tile of two products at once: priced as one product of twice the columns, without the 192-column form, which such tiles do not have.
// The 256x256 tile's price is that of its products alone; with its epilogue it takes 1.13 times that beside a 256x128 tile's (bf16, us, 256x256 and
// 256x128, W [N][K]: 2048 x 5632 x 2048 88 and 82, 3000 x 5400 x 2048 133 and 114, 8192 x 2048 x 768 46 and 53, 20000 x 688 x 256 25 and 28).  The factor is
// taken for every activation, type of C and with G and U kept, too.  All tiles timed beside the chosen one, us: it is the fastest of those four shapes,
// 1024 x 4096 x 4096 and 4096 x 1024 x 512 with silu and G and U kept, none, relu alone, bf16 and fp32 results but for 20000 x 688 x 256 to fp32 (28.4, 24.0 with
// 256x256; kept 44.0, 39.0); of 500 x 2048 x 768 it is up to 1.14 times the fastest (13.2, 11.6 with 64x64; fp32 33.9, 30.0).
gensor_status choose_gated(const GemmView& v, bool vec_ok, const LeadingDims& ld, int64_t strideB, int* out) {
  return remembered({0, v.in_dtype, v.out_dtype, v.bsrc, vec_ok, v.M, v.N, v.K, ld.a, ld.b, ld.c, strideB}, out, [&]() {
    GemmView both = v;
    both.N = 2 * v.N;
    int best = -1;
    double best_us = 1e30;
    for (int i = 0; i < g_num_gated; ++i) {
      const InstanceDesc& d = g_gated[i].d;
      if (!instance_serves(d, v) || (d.vec && !vec_ok) || !offsets_fit(d, v, ld)) continue;
      if (d.direct && !d.any_k() && v.K % d.bk != 0) continue;
      // the second matrix is reached from the first one's base
      const double reach = v.bsrc == B_KC ? (double)(d.bn + 1) * (double)ld.b : (double)(d.bk + 1) * (double)ld.b + d.bn;
      if (((double)strideB + reach) * v.esize >= 2147483647.0) continue;
      const double tiles = (double)((v.M + d.bm - 1) / d.bm) * (double)((2 * v.N + d.bn - 1) / d.bn);
      if (!launch_fits(tiles, d.threads)) continue;
      const double us = fused_price(d, both, 1, false) * (d.alternate() ? 1.13 : 1.0);
      if (us > 0 && us < best_us) { best_us = us; best = i; }
    }
    return best;
  });
}

// The tile of a gradient, whose epilogue takes longer than its products: two values read and two or three stored, an exponential, a reciprocal and some
// thirty operations each, 24 us a round of 256x256 tiles and 0.33 ns an element and unit of smaller ones.  (bf16, us, 256x256, 256x128 and 128x128:
// 8192 x 2048 x 768 49, 56, 65; 3000 x 5400 x 2048 132, 117, 125; 2048 x 5632 x 2048 62, 75, 75; 8192 x 4096 x 4096 254, 297, 364; 1024 x 4096 x 4096 92, 54, 44.
// The prices are those of silu with H in 16 bits, and taken for all.  All tiles timed beside the chosen one: without H and with relu or none within 10 % of
// the fastest as with silu, but for 20000 x 688 x 256 (35.9, 30.3 with 256x256; silu 42.0, 37.0); fp32 operands within 4 %; fp32 results of bf16 operands within 12 %,
// but for 20000 x 688 x 256 (104, 77 with 64x64; relu without H 48, 39).
// Lines of G and U requested under the products did not help: 8192 x 2048 x 768 56, and 69 against 63 among the gradient's other products.)
gensor_status choose_gated_grad(const GemmView& v, bool vec_ok, const LeadingDims& ld, int* out) {
  return remembered({1, v.in_dtype, v.out_dtype, v.bsrc, vec_ok, v.M, v.N, v.K, ld.a, ld.b, ld.c, 0}, out, [&]() {
    int best = -1;
    double best_us = 1e30;
    for (int i = 0; i < g_num_fused; ++i) {
      const InstanceDesc& d = g_fused[i].d;
      if (!g_lm_ends[i].gated_grad || !instance_serves(d, v) || (d.vec && !vec_ok) || !offsets_fit(d, v, ld)) continue;
      if (d.direct && !d.any_k() && v.K % d.bk != 0) continue;
      const double tiles = (double)((v.M + d.bm - 1) / d.bm) * (double)((v.N + d.bn - 1) / d.bn);
      if (!launch_fits(tiles, d.threads)) continue;
      const double price = fused_price(d, v, 1, false), rounds = std::ceil(tiles / gensor_hw_mi355x()->compute_units);
      const double us = price + rounds * (d.alternate() ? 24.0 : d.bm * d.bn * 0.33e-3);
      if (price > 0 && us < best_us) { best_us = us; best = i; }
    }
    return best;
  });
}

template <typename Args>
Args end_args(const GemmView& v, const void* A, int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc, float alpha, const InstanceDesc& d, int columns, int panel) {
  Args a;
  std::memset(&a, 0, sizeof(a));
  a.A = A; a.B = B; a.C = C;
  a.M = (int32_t)v.M; a.N = (int32_t)v.N; a.K = (int32_t)v.K;
  a.lda = lda; a.ldb = ldb; a.ldc = ldc;
  a.alpha = alpha;
  a.split = 1;
  a.tiles_m = (int32_t)((v.M + d.bm - 1) / d.bm);
  a.tiles_n = (int32_t)((v.N + columns - 1) / columns);
  a.batch = 1;
  a.panel = std::min(panel, std::max(1, a.tiles_m));
  a.lds_stages = d.stages;
  return a;
}

// Do two matrices of M x N, `apart` elements from one another, not overlap: one behind the other, or side by side in the same rows?
bool disjoint(int64_t M, int64_t N, int64_t ld, int64_t apart) {
  if (apart >= N && ld - apart >= N) return true;
  return (double)apart >= (double)(M - 1) * (double)ld + (double)N;
}

bool two_pairs(const void* p, int64_t ld, int64_t apart, int64_t N, int osize) { return pairs(p, ld, N, osize) && apart % 2 == 0; }

// Outputs whose rows do not start on cache lines go back through the caches where they are large, as gensor_gemm's do.
bool stored_through(int64_t M, int64_t N, int64_t ld, int osize) {
  return !((ld * osize) % 128 != 0 && M * N * osize > (osize == 2 ? 32ll : 64ll) * 1024 * 1024);
}

gensor_status gated_view(const gensor_problem* p, int32_t act, GemmView* v) {
  if (!p || p->op != GENSOR_OP_GEMM || p->transA != 0 || act < GENSOR_ACT_NONE || act > GENSOR_ACT_SILU) return GENSOR_ERR_INVALID_ARG;
  const gensor_status st = gemm_view(p, v);
  if (st != GENSOR_OK) return st;
  return v->N > (INT32_MAX - 256) / 2 || !extents_fit(*v) ? GENSOR_ERR_UNSUPPORTED : GENSOR_OK;
}

}  // namespace

extern "C" gensor_status gensor_gated_gemm(const gensor_problem* p, int32_t act, float alpha, const void* A, int64_t lda, const void* B, int64_t ldb, int64_t strideB,
                                           const void* bias, void* C, int64_t ldc, void* preact, int64_t ld_preact, int64_t stride_preact, void* hip_stream) {
  return guarded([&]() -> gensor_status {
  GemmView v;
  gensor_status st = gated_view(p, act, &v);
  if (st != GENSOR_OK) return st;
  if (!A || !B || !C || lda < v.K || ldb < (v.bsrc == B_KC ? v.K : v.N) || ldc < v.N || strideB < 0) return GENSOR_ERR_INVALID_ARG;
  if (preact && (ld_preact < v.N || !disjoint(v.M, v.N, ld_preact, stride_preact) || preact == C || (char*)preact + stride_preact * v.osize == C)) return GENSOR_ERR_INVALID_ARG;
  const LeadingDims ld = {lda, ldb, preact ? std::max(ldc, ld_preact) : ldc};
  int tile;
  st = choose_gated(v, vector_ok(v, A, lda, 0, B, ldb, strideB), ld, strideB, &tile);
  if (st == GENSOR_ERR_UNSUPPORTED && v.M >= 1 << 20) {
    // more tiles than a launch can have: the rows in two halves
    gensor_problem half = *p;
    half.M = (v.M / 2 + 255) / 256 * 256;
    // (G and U of a half are as far apart as those of the whole: whether they overlap has been checked)
    st = gensor_gated_gemm(&half, act, alpha, A, lda, B, ldb, strideB, bias, C, ldc, preact, ld_preact, stride_preact, hip_stream);
    if (st != GENSOR_OK) return st;
    const char* A2 = (const char*)A + half.M * lda * v.esize;
    char* C2 = (char*)C + half.M * ldc * v.osize;
    char* Z2 = preact ? (char*)preact + half.M * ld_preact * v.osize : nullptr;
    half.M = v.M - half.M;
    return gensor_gated_gemm(&half, act, alpha, A2, lda, B, ldb, strideB, bias, C2, ldc, Z2, ld_preact, stride_preact, hip_stream);
  }
  if (st != GENSOR_OK) return st;
  const InstanceDesc& d = g_gated[tile].d;
  GatedArgs a = end_args<GatedArgs>(v, A, lda, B, ldb, C, ldc, alpha, d, d.bn / 2, 4);
  a.strideB = strideB;
  a.act = act;
  a.bias = bias;
  a.preact = preact;
  a.ld_preact = ld_preact;
  a.far_preact = stride_preact;
  a.paired = pairs(C, ldc, v.N, v.osize) && (!preact || two_pairs(preact, ld_preact, stride_preact, v.N, v.osize));
  a.through = stored_through(v.M, v.N, ldc, v.osize) && (!preact || stored_through(v.M, v.N, ld_preact, v.osize));
  return launched(g_gated[tile].launch(a, (hipStream_t)hip_stream));
  });
}

extern "C" gensor_status gensor_gated_act_grad(const gensor_problem* p, int32_t act, float alpha, const void* A, int64_t lda, const void* B, int64_t ldb,
                                               const void* preact, int64_t ld_preact, int64_t stride_preact, void* dpreact, int64_t ld_dpreact,
                                               int64_t stride_dpreact, void* H, int64_t ldh, void* hip_stream) {
  return guarded([&]() -> gensor_status {
  GemmView v;
  gensor_status st = gated_view(p, act, &v);
  if (st != GENSOR_OK) return st;
  if (!A || !B || !preact || !dpreact || lda < v.K || ldb < (v.bsrc == B_KC ? v.K : v.N) || (H && ldh < v.N)) return GENSOR_ERR_INVALID_ARG;
  if (ld_preact < v.N || ld_dpreact < v.N || !disjoint(v.M, v.N, ld_preact, stride_preact) || !disjoint(v.M, v.N, ld_dpreact, stride_dpreact)) return GENSOR_ERR_INVALID_ARG;
  const char *g0 = (const char*)preact, *u0 = g0 + stride_preact * v.osize, *dg0 = (const char*)dpreact, *du0 = dg0 + stride_dpreact * v.osize;
  if (g0 == dg0 && (ld_preact != ld_dpreact || stride_preact != stride_dpreact)) return GENSOR_ERR_INVALID_ARG;
  if (g0 == du0 || u0 == dg0 || (H && (H == g0 || H == u0 || H == dg0 || H == du0))) return GENSOR_ERR_INVALID_ARG;
  const LeadingDims ld = {lda, ldb, std::max({ld_preact, ld_dpreact, H ? ldh : (int64_t)0})};
  int tile;
  st = choose_gated_grad(v, vector_ok(v, A, lda, 0, B, ldb, 0), ld, &tile);
  if (st == GENSOR_ERR_UNSUPPORTED && v.M >= 1 << 20) {
    gensor_problem half = *p;
    half.M = (v.M / 2 + 255) / 256 * 256;
    st = gensor_gated_act_grad(&half, act, alpha, A, lda, B, ldb, preact, ld_preact, stride_preact, dpreact, ld_dpreact, stride_dpreact, H, ldh, hip_stream);
    if (st != GENSOR_OK) return st;
    const int64_t h = half.M;
    half.M = v.M - h;
    return gensor_gated_act_grad(&half, act, alpha, (const char*)A + h * lda * v.esize, lda, B, ldb, g0 + h * ld_preact * v.osize, ld_preact, stride_preact,
                                 (char*)dpreact + h * ld_dpreact * v.osize, ld_dpreact, stride_dpreact, H ? (char*)H + h * ldh * v.osize : nullptr, ldh, hip_stream);
  }
  if (st != GENSOR_OK) return st;
  const InstanceDesc& d = g_fused[tile].d;
  GatedArgs a = end_args<GatedArgs>(v, A, lda, B, ldb, H, ldh, alpha, d, d.bn, 2);
  a.act = act;
  a.preact = (void*)preact;
  a.ld_preact = ld_preact;
  a.far_preact = stride_preact;
  a.dpreact = dpreact;
  a.ld_dpreact = ld_dpreact;
  a.far_dpreact = stride_dpreact;
  a.paired = two_pairs(preact, ld_preact, stride_preact, v.N, v.osize) && two_pairs(dpreact, ld_dpreact, stride_dpreact, v.N, v.osize) && (!H || pairs(H, ldh, v.N, v.osize));
  a.through = stored_through(v.M, v.N, ld_dpreact, v.osize) && (!H || stored_through(v.M, v.N, ldh, v.osize));
  return launched(g_lm_ends[tile].gated_grad(a, (hipStream_t)hip_stream));
  });
}

// ------------------------------------------------------------------------------------ scores of a vocabulary
namespace gensor {

// Sums of exponentials relative to a maximum, and weighted with the exponents: joined with another part's (join_sums).  A part without terms has the
// maximum -inf and the sums 0.
__device__ inline void join_scores(float& top, float& sum, float& rest, float top2, float sum2, float rest2) {
  constexpr float log2e = 1.44269504088896340736f;
  const float both = fmaxf(top, top2), r = lse_reference(both);
  const float d1 = fabsf(top) == INFINITY ? 0.f : top - r, d2 = fabsf(top2) == INFINITY ? 0.f : top2 - r;
  const float f1 = __builtin_amdgcn_exp2f(log2e * d1), f2 = __builtin_amdgcn_exp2f(log2e * d2);
  // (terms that vanish beside the larger maximum: the distance itself may be infinite)
  rest = (f1 > 0.f ? f1 * fmaf(sum, d1, rest) : 0.f) + (f2 > 0.f ? f2 * fmaf(sum2, d2, rest2) : 0.f);
  sum = sum * f1 + sum2 * f2;
  top = both;
}

// (the last of a part's four values is not used, and not read: its register would be another's before it arrives)
typedef float f32x3 __attribute__((ext_vector_type(3)));

struct AdvanceArgs {
  const f32x4* parts;              // of this piece
  const float* set_max;
  const float* logits;
  int32_t slabs, slab_pitch, sets, set_pitch, set_size;
  int32_t token_first, tokens, row_first, vocab, top, first, last;
  f32x4* state;                    // [tokens]: joined so far
  float* bar;                      // [tokens]: a later logit is among the largest only above it
  float* values;                   // [tokens][top]: the largest logits so far; log probabilities in the end
  int64_t* index;
  const int64_t* targets;          // (memory that may be read, too, where logprob is NULL)
  int64_t ignore;
  const float* at_target;
  float *logprob, *lse, *entropy;
};

// x of all lanes joined (by an operation whose operands may be swapped): all of them hold the result.  In registers, without LDS.
template <typename Op>
__device__ inline float over_lanes(float x, Op&& op) {
  auto moved = [&](auto ctrl_tag) { return as_f32((uint32_t)__builtin_amdgcn_mov_dpp((int)as_u32(x), decltype(ctrl_tag)::value, 0xF, 0xF, true)); };
  x = op(x, moved(std::integral_constant<int, 0xB1>{}));               // quad_perm [1,0,3,2]
  x = op(x, moved(std::integral_constant<int, 0x4E>{}));               // quad_perm [2,3,0,1]
  x = op(x, moved(std::integral_constant<int, 0x141>{}));              // row_half_mirror
  x = op(x, moved(std::integral_constant<int, 0x140>{}));              // row_mirror
  return over_groups<16>(x, op);
}

// Parts (maximum, sum, weighted sum), a lane each, joined: all lanes hold the result.
__device__ inline void join_lanes(float& top, float& sum, float& rest) {
  constexpr float log2e = 1.44269504088896340736f;
  auto plus = [](float x, float y) { return x + y; };
  const float all = over_lanes(top, [](float x, float y) { return fmaxf(x, y); });
  const float d = fabsf(top) == INFINITY ? 0.f : top - lse_reference(all), f = __builtin_amdgcn_exp2f(log2e * d);
  rest = over_lanes(f > 0.f ? f * fmaf(sum, d, rest) : 0.f, plus);
  sum = over_lanes(sum * f, plus);
  top = all;
}

// A number that n of the lanes' values (COUNT each) reach (nth_reached: twenty ballots a value; counting for each value those above it takes three
// instructions a lane)
template <int COUNT>
__device__ inline float nth_of_lanes(const float (&x)[COUNT], int n) {
  uint32_t key[COUNT];
#pragma unroll
  for (int c = 0; c < COUNT; ++c) key[c] = (uint32_t)(rank_key(x[c], 0) >> 32);
  return nth_reached(n, [&](uint32_t least) __attribute__((always_inline)) {
    int reach = 0;
#pragma unroll
    for (int c = 0; c < COUNT; ++c) reach += (int)__popcll(__ballot(key[c] >= least));
    return reach;
  });
}

// WAVES waves per token join a piece's parts to what was joined before, and find the largest logits among the piece's and those so far.
//
// The search.  A bar that no more than a few logits reach is known before any is read: what the pieces so far say (the top'th largest, to be
// exceeded), and the top'th largest of 64 maxima of disjoint groups of this piece's sets (to be reached; sought only where it may be the higher one, mostly in the
// first two pieces: 4096 tokens' second 21 us without, 13 with).  Sets whose maximum does not reach it hold none of the largest; the logits of the others
// that reach it, and the largest so far, are gathered in LDS, and each one's place is the number of those above it: no order in which anything is gathered
// matters.  (Putting them into a sorted list, a lane each, one by one took 0.3 us apiece: 23 us for one token's five, 43 for the twenty of 301 tokens.)
// Where more come up than there is room for -- many equal ones, as of a padded batch's tokens of zeros -- all that were kept are looked through in their
// order.
//
// Bound by a chain of loads (parts and maxima, then the sets) and by the vector unit.  us: one token's five of 50257 (8 waves) 4.9, 301 tokens' twenty of
// 5003 (4 waves) 6.6, 4096 tokens' eight (a wave each) 9 to 11 a piece, without alternatives 6.6.  (With the tokens in a loop, whose constants take registers:
// 154 in place of 67, three workgroups a unit where there is work for four, 13 a piece.)
template <int WAVES, bool TOP>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void advance_kernel(const AdvanceArgs a) {
  constexpr int TOKENS = WAVES == 1 ? 4 : 1, AHEAD = WAVES == 1 ? 12 : 8, KEYS = WAVES == 1 ? 512 : 1024, SETS = 512, GROUPS = 4;
  __shared__ float joined[TOKENS][WAVES == 1 ? 1 : 3 * WAVES];
  __shared__ float group_max[WAVES == 1 ? 1 : WAVES][64];
  __shared__ int set_list[TOKENS][SETS];
  __shared__ uint64_t keys[TOKENS][KEYS];
  __shared__ int counts[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = WAVES == 1 ? 0 : wave, at = WAVES == 1 ? wave : 0;
  auto meet = [&]() {
    if constexpr (WAVES > 1) __syncthreads();
    else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
  // places in a list for the lanes that have something; the count goes on beyond what there is room for
  int own_counts[2] = {0, 0};
  auto places = [&](int which, bool mine) -> int {
    const uint64_t all = __ballot(mine);
    if (all == 0) return 0;
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0u));
    if constexpr (WAVES == 1) {
      const int first = own_counts[which];
      own_counts[which] = first + (int)__popcll(all);
      return first + before;
    }
    int first = 0;
    if (lane == 0) first = atomicAdd(&counts[which], (int)__popcll(all));
    return __builtin_amdgcn_readfirstlane(first) + before;
  };
  auto count = [&](int which) { return WAVES == 1 ? own_counts[which] : counts[which]; };
  const int t = a.token_first + blockIdx.x * TOKENS + (WAVES == 1 ? wave : 0);
  if (t >= a.tokens) return;
  // everything that is known where to find is asked for first, and without a condition: what is not there is replaced afterwards
  const float* set_max = a.set_max + (int64_t)t * a.set_pitch;
  const float* logits = a.logits + (int64_t)t * a.set_pitch * a.set_size;
  float* values = a.values + (int64_t)t * a.top;
  int64_t* index = a.index + (int64_t)t * a.top;
  const f32x4* parts = a.parts + (int64_t)t * a.slab_pitch;
  f32x3 p[4];
  auto ask = [&](int s) {
#pragma unroll
    for (int u = 0; u < 4; ++u) p[u] = *(const f32x3*)(parts + min(s + 64 * WAVES * u, a.slabs - 1));
  };
  ask(64 * part + lane);
  const f32x3 so_far = *(const f32x3*)(a.state + t);
  const int64_t target = a.targets[t];
  const float at_target = a.at_target[t];
  float m[AHEAD], most[GROUPS], own_value = 0.f, bar = NAN;
  int64_t own_entry = -1;
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) most[g] = -INFINITY;
  auto ask_sets = [&](int s) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) m[u] = set_max[min(s + 64 * WAVES * u, a.sets - 1)];
  };
  auto set_there = [&](int s) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s + 64 * WAVES * u >= a.sets) m[u] = -INFINITY;
  };
  if constexpr (TOP) {
    ask_sets(64 * part + lane);
    bar = a.bar[t];
    own_value = values[min(lane, a.top - 1)];
    own_entry = index[min(lane, a.top - 1)];
  }
  float top = -INFINITY, sum = 0.f, rest = 0.f;
  for (int s0 = 64 * part; s0 < a.slabs; s0 += 4 * 64 * WAVES) {
    if (s0 != 64 * part) ask(s0 + lane);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s0 + lane + 64 * WAVES * u >= a.slabs) p[u] = f32x3{-INFINITY, 0.f, 0.f};
    // (four parts to one reference)
    const float both = fmaxf(fmaxf(fmaxf(p[0][0], p[1][0]), fmaxf(p[2][0], p[3][0])), top), r = lse_reference(both);
    auto scaled = [&](float part_top, float part_sum, float part_rest, float& to_sum, float& to_rest) {
      const float d = fabsf(part_top) == INFINITY ? 0.f : part_top - r, f = __builtin_amdgcn_exp2f(1.44269504088896340736f * d);
      to_rest += f > 0.f ? f * fmaf(part_sum, d, part_rest) : 0.f;
      to_sum += part_sum * f;
    };
    float new_sum = 0.f, new_rest = 0.f;
    scaled(top, sum, rest, new_sum, new_rest);
#pragma unroll
    for (int u = 0; u < 4; ++u) scaled(p[u][0], p[u][1], p[u][2], new_sum, new_rest);
    top = both; sum = new_sum; rest = new_rest;
  }
  if constexpr (TOP) {
    set_there(64 * part + lane);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) most[u % GROUPS] = fmaxf(most[u % GROUPS], m[u]);
#pragma unroll 4
    for (int s = 64 * (part + WAVES * AHEAD) + lane; s < a.sets; s += 64 * WAVES) most[0] = fmaxf(most[0], set_max[s]);
    if (a.first || lane >= a.top) own_entry = -1;
    if (a.first) bar = NAN;
  }
  join_lanes(top, sum, rest);
  if (WAVES > 1 && threadIdx.x < 2) counts[threadIdx.x] = 0;
  if constexpr (WAVES > 1) {
    if constexpr (TOP) {
      group_max[wave][lane] = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
    }
    if (lane == 0) {
      joined[0][3 * wave] = top;
      joined[0][3 * wave + 1] = sum;
      joined[0][3 * wave + 2] = rest;
    }
    meet();
    top = lane < WAVES ? joined[0][3 * lane] : -INFINITY;
    sum = lane < WAVES ? joined[0][3 * lane + 1] : 0.f;
    rest = lane < WAVES ? joined[0][3 * lane + 2] : 0.f;
    join_lanes(top, sum, rest);
    if constexpr (TOP) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) most[g] = -INFINITY;
#pragma unroll
      for (int v = 0; v < WAVES; ++v) most[v % GROUPS] = fmaxf(most[v % GROUPS], group_max[v][lane]);
    }
  } else {
    meet();
  }
  if (!a.first) {
    float x = so_far[0], y = so_far[1], z = so_far[2];
    join_scores(x, y, z, top, sum, rest);
    top = x; sum = y; rest = z;
  }
  const float ref = lse_reference(top), log_sum = logf(sum);
  if (part == 0 && lane == 0) {
    if (!a.last) {
      a.state[t] = f32x4{top, sum, rest, 0.f};
    } else {
      if (a.lse) a.lse[t] = ref + log_sum;
      if (a.entropy) a.entropy[t] = log_sum - rest / sum;
      if (a.logprob) {
        // (the maximum's part first: a target that is the maximum loses log(1 + the others), not a difference of large numbers)
        a.logprob[t] = target == a.ignore ? 0.f : target >= 0 && target < a.vocab ? (at_target - ref) - log_sum : NAN;
      }
    }
  }
  if constexpr (!TOP) return;

  // ---- sets that reach the bar; all of them are stored (least_wanted)
  // (many are sought among more groups, of which fewer hold two of them)
  float least;
  if (a.top > 24) {
    int above = 0;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) above += (int)__popcll(__ballot(most[g] > bar));
    least = least_wanted(bar, above >= a.top, [&]() { return nth_of_lanes(most, a.top); });
  } else {
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) most[0] = fmaxf(most[0], most[g]);
    least = least_wanted(bar, (int)__popcll(__ballot(most[0] > bar)) >= a.top, [&]() { return nth_of_lanes<1>({most[0]}, a.top); });
  }
  auto reaches = [&](float v) { return v >= least; };
  for (int s0 = 64 * part; s0 < a.sets; s0 += 64 * WAVES * AHEAD) {
    if (s0 != 64 * part) {
      ask_sets(s0 + lane);
      set_there(s0 + lane);
    }
    uint32_t hits = 0;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) hits |= reaches(m[u]) && s0 + lane + 64 * WAVES * u < a.sets ? 1u << u : 0u;
    while (__any(hits != 0)) {
      const int to = places(0, hits != 0);
      if (hits != 0 && to < SETS) set_list[at][to] = s0 + lane + 64 * WAVES * __builtin_ctz(hits);
      hits &= hits - 1;
    }
  }
  // the largest so far
  const uint64_t own_key = own_entry >= 0 ? rank_key(own_value, (int)own_entry) : 0;
  if (!a.first && part == 0) {
    const int to = places(1, own_key != 0);
    if (own_key) keys[at][to] = own_key;
  }
  meet();
  // ---- their logits that reach it
  const int size = a.set_size, per = 64 / size;                      // sets that a wave looks at together
  auto logit = [&](int set, int& entry) -> float {
    entry = set * size + lane % size;
    return logits[(int64_t)set * size + lane % size];
  };
  const int n_sets = count(0);
  if (n_sets <= SETS) {
    for (int j = part * per; j < n_sets; j += 4 * per * WAVES) {
      float v[4];
      int e[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int which = j + u * per * WAVES + lane / size;
        e[u] = 0;
        v[u] = which < n_sets ? logit(set_list[at][which], e[u]) : NAN;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool mine = reaches(v[u]) && e[u] < a.vocab - a.row_first;
        const int to = places(1, mine);
        if (mine && to < KEYS) keys[at][to] = rank_key(v[u], a.row_first + e[u]);
      }
    }
  }
  meet();
  const int n = count(1);
  auto put = [&](int rank, uint64_t key) {
    index[rank] = key ? (int64_t)key_entry(key) : -1;
    values[rank] = !key ? NAN : a.last ? (key_value(key) - ref) - log_sum : key_value(key);
    if (rank == a.top - 1 && !a.last) a.bar[t] = key ? key_value(key) : NAN;
  };
  if (n_sets <= SETS && n <= KEYS) {
    for (int i = 64 * part + lane; i < n; i += 64 * WAVES) {
      const uint64_t own = keys[at][i];
      int rank = 0;
#pragma unroll 4
      for (int o = 0; o < n; ++o) rank += keys[at][o] > own;
      if (rank < a.top) put(rank, own);
    }
    for (int i = n + 64 * part + lane; i < a.top; i += 64 * WAVES) put(i, 0);
    return;
  }
  // ---- too many: set after set in the order of their entries, and as often as there might be no room for more, those that are not among the largest
  // go, after which only larger logits are taken (an equal one's entry is higher)
  constexpr int ROOM = (KEYS - GENSOR_TOP_MAX) / (64 * WAVES), AT_ONCE = ROOM < 4 ? ROOM : 4, OWN = KEYS / (64 * WAVES);
  static_assert(AT_ONCE >= 1 && OWN >= 1, "room for what is looked at together");
  auto only_largest = [&](int m) -> int {
    uint64_t own[OWN];
    int rank[OWN];
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
      const int i = 64 * (part + WAVES * k) + lane;
      own[k] = i < m ? keys[at][i] : 0;
      rank[k] = 0;
    }
#pragma unroll 4
    for (int o = 0; o < m; ++o) {
      const uint64_t other = keys[at][o];
#pragma unroll
      for (int k = 0; k < OWN; ++k) rank[k] += other > own[k];
    }
    meet();
    const int left = min(m, a.top);
#pragma unroll
    for (int k = 0; k < OWN; ++k)
      if (own[k] && rank[k] < left) keys[at][rank[k]] = own[k];
    own_counts[1] = left;
    if (WAVES > 1 && threadIdx.x == 0) counts[1] = left;
    meet();
    return left;
  };
  meet();                                                            // (everyone has read the counts)
  own_counts[1] = 0;
  if (WAVES > 1 && threadIdx.x == 0) counts[1] = 0;
  meet();
  if (!a.first && part == 0) {
    const int to = places(1, own_key != 0);
    if (own_key) keys[at][to] = own_key;
  }
  float taken = least;
  constexpr int CHUNK = 64 * WAVES;
  for (int c0 = 0; c0 < a.sets; c0 += CHUNK) {
    // (sets none of which holds one are passed over together)
    const int own_set = c0 + 64 * part + lane;
    const float own_max = own_set < a.sets ? set_max[own_set] : NAN;
    auto some = [&]() { return WAVES > 1 ? __syncthreads_or(own_max >= taken) != 0 : __any(own_max >= taken) != 0; };
    if (!some()) continue;
    for (int s0 = c0; s0 < min(c0 + CHUNK, a.sets); s0 += AT_ONCE * per * WAVES) {
      meet();
      const int so_many = count(1);
      meet();
      if (so_many > KEYS - AT_ONCE * 64 * WAVES) {
        only_largest(so_many);                                       // (more than GENSOR_TOP_MAX: `top` are left)
        const float next = next_above(key_value(keys[at][a.top - 1]));
        if (!(next <= taken)) taken = next;
        if (!some()) break;
      }
      float v[AT_ONCE];
      int e[AT_ONCE];
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const int set = s0 + (part + u * WAVES) * per + lane / size;
        e[u] = 0;
        v[u] = set < min(c0 + CHUNK, a.sets) && set_max[set] >= taken ? logit(set, e[u]) : NAN;
      }
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const bool mine = v[u] >= taken && e[u] < a.vocab - a.row_first;
        const int to = places(1, mine);
        if (mine) keys[at][to] = rank_key(v[u], a.row_first + e[u]);
      }
    }
  }
  meet();
  const int so_many = count(1);
  meet();
  const int left = only_largest(so_many);
  for (int i = 64 * part + lane; i < a.top; i += 64 * WAVES) put(i, i < left ? keys[at][i] : 0);
}

}  // namespace gensor

namespace {

// Logits of a piece at most, where the largest are asked for.  (4096 tokens over 50257 entries, eight alternatives, f16, us: 128 MiB 355, 256 327, 384 316,
// 512 320, 1024 311.)
const size_t kScoreBytes = (size_t)384 << 20;
// ... of which a first piece that may keep them all
const size_t kHeadBytes = (size_t)32 << 20;

struct ScorePlan {
  int64_t slabs, sets;             // of a piece
  size_t parts, maxima, logits;    // bytes
  size_t total() const { return parts + maxima + logits; }
};

ScorePlan score_plan(const InstanceDesc& d, int64_t T, int64_t rows, int top) {
  ScorePlan s;
  const int set = score_set(d.wm);
  s.slabs = (rows + d.wm - 1) / d.wm;
  s.sets = top ? s.slabs * (d.wm / set) : 0;
  s.parts = round_up((size_t)(s.slabs * T) * 16, 256);
  s.maxima = round_up((size_t)(s.sets * T) * 4, 256);
  s.logits = round_up((size_t)(s.sets * T) * set * 4, 256);
  return s;
}

// [state][bar][logit of the target] in front of a piece's
size_t score_head(int64_t T) { return round_up((size_t)T * 16, 256) + 2 * round_up((size_t)T * 4, 256); }

// Vocabulary entries of a piece where the room does not limit it
int64_t score_piece(const InstanceDesc& d, int64_t T, int64_t V, int top) {
  if (top == 0) return V;
  const int64_t most = std::max<int64_t>(1, (int64_t)(kScoreBytes / ((size_t)T * 4)) / d.bm) * d.bm;
  return std::min(V, most);
}

gensor_status choose_score(int dtype, int64_t T, int64_t V, int64_t D, const void* W, int64_t ldw, const void* X, int64_t ldx, FusedChoice* c) {
  const GemmView v = prob_view(dtype, V, T, D);
  const LeadingDims ld = {ldw, ldx, 0};
  return choose(v, FUSED_LSE, vector_ok(v, W, ldw, 0, X, ldx, 0), ld, 0, c);
}

size_t score_bytes(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, int top) {
  const GemmView v = prob_view(dtype, V, T, D);
  size_t most = 0;
  for (int vec = 0; vec < 2; ++vec) {
    FusedChoice c;
    const LeadingDims ld = {D, D, 0};
    if (choose(v, FUSED_LSE, vec != 0, ld, 0, &c) == GENSOR_OK) most = std::max(most, score_plan(c.f->d, T, score_piece(c.f->d, T, V, top), top).total());
  }
  // (rows so far apart that another tile serves them: a piece of any)
  for (int i = 0; i < g_num_fused; ++i) {
    const InstanceDesc& d = g_fused[i].d;
    if (g_lm_ends[i].score && instance_serves(d, v)) most = std::max(most, score_plan(d, T, std::min<int64_t>(V, d.bm), top).total());
  }
  return score_head(T) + most;
}

struct ScoreOutputs {
  float *logprob, *lse, *entropy;
  int32_t top;
  int64_t* top_index;
  float* top_logprob;
};

gensor_status run_scores(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx, const void* W, int64_t ldw, float scale,
                         const int64_t* targets, int64_t ignore, const ScoreOutputs& out, void* workspace, size_t workspace_bytes, hipStream_t s) {
  FusedChoice c;
  gensor_status st = choose_score(dtype, T, V, D, W, ldw, X, ldx, &c);
  if (st == GENSOR_ERR_UNSUPPORTED && T >= 1 << 20) {
    // more tiles than a launch can have: the tokens in two halves
    const int64_t half = (T / 2 + 255) / 256 * 256;
    st = run_scores(dtype, half, V, D, X, ldx, W, ldw, scale, targets, ignore, out, workspace, workspace_bytes, s);
    if (st != GENSOR_OK) return st;
    auto behind = [&](float* p) { return p ? p + half : nullptr; };
    const ScoreOutputs rest = {behind(out.logprob), behind(out.lse), behind(out.entropy), out.top, out.top ? out.top_index + half * out.top : nullptr,
                               out.top ? out.top_logprob + half * out.top : nullptr};
    return run_scores(dtype, T - half, V, D, (const char*)X + half * ldx * size_of(dtype), ldx, W, ldw, scale, targets ? targets + half : nullptr, ignore, rest,
                      workspace, workspace_bytes, s);
  }
  if (st != GENSOR_OK) return st;
  const InstanceDesc& d = c.f->d;
  const size_t room = usable_room(workspace, workspace_bytes), head = score_head(T);
  int64_t piece = score_piece(d, T, V, out.top);
  while (head + score_plan(d, T, piece, out.top).total() > room) {
    if (piece <= d.bm) return GENSOR_ERR_WORKSPACE;
    piece = std::max<int64_t>(1, piece / 2 / d.bm) * d.bm;
  }
  // Nothing is known of the first piece's logits, so all of them are kept: it is one round of tiles, after which few are above a token's bar.  Where all are
  // two rounds, or few bytes, there is one piece.  (Eight alternatives, f16, us, in one piece and in two: 512 tokens over 50257 entries 69, 72; 4096 over 5000
  // 65, 72; 2.3 rounds, 640 over 50257, 94, 86.)
  int64_t rows = piece;
  if (out.top) {
    const int64_t tiles_n = (T + d.bn - 1) / d.bn, units = gensor_hw_mi355x()->compute_units;
    if (piece * T * 4 > (int64_t)kHeadBytes && (piece + d.bm - 1) / d.bm * tiles_n > 2 * units) rows = std::min(piece, std::max<int64_t>(1, units / tiles_n) * d.bm);
    // The others are whole rounds, where that makes them no more: a launch's last round leaves units idle.  (3000 tokens over 50257 entries 265 us without, 246 with.)
    const int64_t whole = piece / d.bm * tiles_n / units * units / tiles_n * d.bm, rest = V - rows;
    if (whole > 0 && (rest + whole - 1) / whole == (rest + piece - 1) / piece) piece = whole;
  }
  const ScorePlan pl = score_plan(d, T, std::max(rows, piece), out.top);
  char* at = (char*)workspace;
  f32x4* state = (f32x4*)at;
  float* bar = (float*)(at + round_up((size_t)T * 16, 256));
  float* at_target = (float*)((char*)bar + round_up((size_t)T * 4, 256));
  f32x4* parts = (f32x4*)(at + head);
  float* maxima = (float*)(at + head + pl.parts);
  float* logits = (float*)(at + head + pl.parts + pl.maxima);
  for (int64_t entry = 0; entry < V; entry += rows, rows = piece) {
    rows = std::min(rows, V - entry);
    const bool first = entry == 0, last = entry + rows == V;
    const GemmView q = prob_view(dtype, rows, T, D);
    ScoreArgs a = end_args<ScoreArgs>(q, (const char*)W + entry * ldw * size_of(dtype), ldw, X, ldx, nullptr, 0, scale, d, d.bn, 4);
    a.targets = out.logprob ? targets : nullptr;
    a.ignore = ignore;
    a.tokens = (int32_t)T;
    a.row_first = (int32_t)entry;
    a.vocab = (int32_t)V;
    a.weighted = out.entropy != nullptr;
    a.slabs = (int32_t)pl.slabs;
    a.sets = (int32_t)pl.sets;
    a.parts = parts;
    a.set_max = maxima;
    a.logits = logits;
    a.bar = first ? nullptr : bar;
    a.at_target = at_target;
    if (g_lm_ends[c.f - g_fused].score(a, s) != hipSuccess) return GENSOR_ERR_DEVICE;
    AdvanceArgs v;
    std::memset(&v, 0, sizeof(v));
    v.parts = parts;
    v.set_max = maxima;
    v.logits = logits;
    v.slabs = (int32_t)((rows + d.wm - 1) / d.wm);
    v.slab_pitch = a.slabs;
    v.set_size = score_set(d.wm);
    v.sets = out.top ? (int32_t)((rows + v.set_size - 1) / v.set_size) : 0;
    v.set_pitch = a.sets;
    v.tokens = (int32_t)T;
    v.row_first = (int32_t)entry;
    v.vocab = (int32_t)V;
    v.top = out.top;
    v.first = first;
    v.last = last;
    v.state = state;
    v.bar = bar;
    v.values = out.top_logprob;
    v.index = out.top_index;
    v.targets = out.logprob ? targets : (const int64_t*)state;
    v.ignore = ignore;
    v.at_target = at_target;
    v.logprob = out.logprob;
    v.lse = out.lse;
    v.entropy = out.entropy;
    // (waves do part of the work over again.  The whole call over 50257 entries, us, eight alternatives and fifty, with 1, 4 and 8 waves: one token 24.4, 21.7,
    // 21.9 and 32.1, 24.7, 24.1; 256 tokens 39.7, 36.6, 36.6 and 50.0, 39.9, 39.0; 1024 109.6, 110.2, 113.2 and 129, 120, 124; 4096 312, 332, 358 and 356, 375, 415)
    auto advance = [&](auto with_top) {
      constexpr bool TOP = decltype(with_top)::value;
      if (T <= 256) hipLaunchKernelGGL((advance_kernel<8, TOP>), dim3((unsigned)T), dim3(512), 0, s, v);
      else if (T <= 1024) hipLaunchKernelGGL((advance_kernel<4, TOP>), dim3((unsigned)T), dim3(256), 0, s, v);
      else
        for (int64_t t = 0; t < T; t += 4 << 20) {
          v.token_first = (int32_t)t;
          hipLaunchKernelGGL((advance_kernel<1, TOP>), dim3((unsigned)((std::min<int64_t>(T - t, 4 << 20) + 3) / 4)), dim3(256), 0, s, v);
        }
    };
    if (out.top) advance(std::true_type{});
    else advance(std::false_type{});
    if (hipGetLastError() != hipSuccess) return GENSOR_ERR_DEVICE;
  }
  return GENSOR_OK;
}

bool valid_scale(float scale) { return scale > 0.f && std::isfinite(scale); }

}  // namespace

extern "C" size_t gensor_logprobs_workspace_bytes(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, int32_t top) {
  size_t bytes = 0;
  guarded([&]() -> gensor_status {
    if (check_xent(dtype, T, V, D) == GENSOR_OK && top >= 0 && top <= GENSOR_TOP_MAX && top <= V) bytes = score_bytes(dtype, T, V, D, top);
    return GENSOR_OK;
  });
  return bytes;
}

extern "C" gensor_status gensor_logprobs(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx, const void* W, int64_t ldw, float scale,
                                         const int64_t* targets, int64_t ignore_index, float* logprob, float* lse, float* entropy, int32_t top, int64_t* top_index,
                                         float* top_logprob, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> gensor_status {
  const gensor_status st = check_xent(dtype, T, V, D);
  if (st != GENSOR_OK) return st;
  if (!X || !W || ldx < D || ldw < D || !valid_scale(scale) || top < 0 || top > GENSOR_TOP_MAX || top > V) return GENSOR_ERR_INVALID_ARG;
  if ((!logprob && !lse && !entropy && !top) || (logprob && !targets) || (targets && !aligned(targets, 8))) return GENSOR_ERR_INVALID_ARG;
  if (top ? (!top_index || !top_logprob || !aligned(top_index, 8)) : (top_index || top_logprob)) return GENSOR_ERR_INVALID_ARG;
  const ScoreOutputs out = {logprob, lse, entropy, top, top_index, top_logprob};
  return run_scores(dtype, T, V, D, X, ldx, W, ldw, scale, targets, ignore_index, out, workspace, workspace_bytes, (hipStream_t)hip_stream);
  });
}

// ------------------------------------------------------------------------------------ learning from a teacher
namespace gensor {

struct TeacherArgs {
  const char* X;
  const char* W;
  int64_t ldx, ldw;
  const int64_t* index;
  const float* teacher;
  const float* lse;
  int32_t T, V, D, k, normalize;
  float scale;
  float* loss;                     // forward
  const float* dloss;              // gradient
  float* weights;                  // dloss * scale * P, zero for tokens that teach nothing
  int32_t* entries;                // [T][k]: where G gets another value, or -1
  float* values;                   // ... and that value
};

// A token's entries, probabilities and logits in LDS.
struct TeacherEntries {
  int entry[256];
  float log_p[256], p[256], z[256];
  float mass;
  int bad;
};

// Fills them, all 256 threads of a workgroup: a wave takes four entries at a time, whose rows of W it reads side by side with the token's row of X, two
// vectors a lane of each requested together.  Bound by those rows, from the last-level cache: 4096 tokens' sixteen entries of width 768 in 16 bits are 100 MB,
// 17.5 us (5.7 TB/s; one vector ahead 21.3), with the gradient's values 20 to 21.
template <typename T, bool VEC>
__device__ inline void teacher_entries(const TeacherArgs& a, int t, TeacherEntries& e) {
  constexpr int ES = ElemSize<T>::value, EPC = 16 / ES;
  const int i = threadIdx.x, lane = i & 63, wave = __builtin_amdgcn_readfirstlane(i >> 6);
  auto plus = [](float x, float y) { return x + y; };
  __syncthreads();                                                   // (the token before)
  if (i == 0) e.bad = 0;
  __syncthreads();
  if (i < a.k) {
    const int64_t at = a.index[(int64_t)t * a.k + i];
    const float q = a.teacher[(int64_t)t * a.k + i];
    const bool there = at >= 0 && at < a.V;
    e.entry[i] = there ? (int)at : -1;
    if (at < -1 || at >= a.V) e.bad = 1;                             // (any of the threads that find one)
    e.log_p[i] = there ? q : -INFINITY;
  }
  __syncthreads();
  const char* x = a.X + (int64_t)t * a.ldx * ES;
  for (int j = 4 * wave; j < a.k; j += 16) {
    const char* w[4];
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 4; ++u) w[u] = a.W + (int64_t)(j + u < a.k ? max(e.entry[j + u], 0) : 0) * a.ldw * ES;
    if constexpr (VEC) {
      for (int c = lane * EPC; c < a.D; c += 2 * 64 * EPC) {
        const int c2 = c + 64 * EPC;
        u32x4 xv[2], wv[4][2];
        xv[0] = *(const u32x4*)(x + (int64_t)c * ES);
        xv[1] = c2 < a.D ? *(const u32x4*)(x + (int64_t)c2 * ES) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          wv[u][0] = *(const u32x4*)(w[u] + (int64_t)c * ES);
          wv[u][1] = c2 < a.D ? *(const u32x4*)(w[u] + (int64_t)c2 * ES) : u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int n = 0; n < EPC; ++n) {
              if constexpr (ES == 4) acc[u] = fmaf(as_f32(xv[h][n]), as_f32(wv[u][h][n]), acc[u]);
              else acc[u] = fmaf(from_pair<T>(xv[h][n / 2], n & 1), from_pair<T>(wv[u][h][n / 2], n & 1), acc[u]);
            }
      }
    } else {
      for (int c = lane; c < a.D; c += 4 * 64) {
        float xv[4], wv[4][4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const bool there = c + 64 * h < a.D;
          xv[h] = there ? to_float<T>(x, c + 64 * h) : 0.f;
#pragma unroll
          for (int u = 0; u < 4; ++u) wv[u][h] = there ? to_float<T>(w[u], c + 64 * h) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int h = 0; h < 4; ++h) acc[u] = fmaf(xv[h], wv[u][h], acc[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float z = over_lanes(acc[u], plus);
      if (lane == 0 && j + u < a.k) e.z[j + u] = a.scale * z;
    }
  }
  if (wave == 3) {                                                   // (it has the fewest entries)
    float shift = 0.f;
    if (a.normalize) {
      float top = -INFINITY, sum = 0.f;
      for (int j = lane; j < a.k; j += 64) {
        if (e.entry[j] >= 0) e.log_p[j] *= a.scale;
        top = fmaxf(top, e.log_p[j]);
      }
      top = over_lanes(top, [](float x, float y) { return fmaxf(x, y); });
      if (top > -INFINITY)
        for (int j = lane; j < a.k; j += 64) sum += expf(e.log_p[j] - top);
      shift = top > -INFINITY ? top + logf(over_lanes(sum, plus)) : 0.f;
    }
    float mass = 0.f;
    for (int j = lane; j < a.k; j += 64) {
      const float q = e.log_p[j] - shift;
      e.log_p[j] = q;
      e.p[j] = expf(q);
      mass += e.p[j];
    }
    mass = over_lanes(mass, plus);
    if (lane == 0) e.mass = mass;
  }
  __syncthreads();
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void teacher_loss_kernel(const TeacherArgs a) {
  __shared__ TeacherEntries e;
  for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
    teacher_entries<T, VEC>(a, t, e);
    if (threadIdx.x >= 64) continue;
    const float lse = a.lse[t];
    float loss = 0.f;
    // (entries that are none and probabilities of zero by choice: their logarithms and logits may be infinite)
    for (int j = threadIdx.x; j < a.k; j += 64) loss += e.p[j] == 0.f ? 0.f : e.p[j] * ((e.log_p[j] - e.z[j]) + lse);
    loss = over_lanes(loss, [](float x, float y) { return x + y; });
    if (threadIdx.x == 0) a.loss[t] = e.bad ? NAN : loss;
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void teacher_weights_kernel(const TeacherArgs a) {
  __shared__ TeacherEntries e;
  for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
    teacher_entries<T, VEC>(a, t, e);
    const float dloss = a.dloss[t] * a.scale;
    const bool teaches = !e.bad && e.mass != 0.f && dloss != 0.f;
    if (threadIdx.x == 0) a.weights[t] = teaches ? dloss * e.mass : 0.f;
    const int j = threadIdx.x;
    if (j < a.k) {
      // an entry that is named again is the first one's business
      const int at = e.entry[j];
      bool mine = teaches && at >= 0;
      float p = 0.f;
      if (mine)
        for (int i = 0; i < a.k; ++i)
          if (e.entry[i] == at) {
            if (i < j) mine = false;
            p += e.p[i];
          }
      a.entries[(int64_t)t * a.k + j] = mine ? at : -1;
      a.values[(int64_t)t * a.k + j] = mine ? dloss * (e.mass * expf(e.z[j] - a.lse[t]) - p) : 0.f;
    }
  }
}

// scale[0]: a power of two's worth of G, so that the largest weight becomes 2^15 (xent_scale_kernel says why); scale[1]: its inverse
__global__ __launch_bounds__(1024) void teacher_scale_kernel(const float* weights, int tokens, float* scale) {
  constexpr int UNROLL = 8;
  __shared__ float tops[16];
  float top = 0.f;
  for (int first = threadIdx.x; first < tokens; first += UNROLL * 1024) {
    float x[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) x[u] = first + u * 1024 < tokens ? fabsf(weights[first + u * 1024]) : 0.f;
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
      if (x[u] < INFINITY) top = fmaxf(top, x[u]);
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

// G of a piece at the teacher's entries
template <typename T>
__global__ __launch_bounds__(256) void teacher_place_kernel(const int32_t* entries, const float* values, const float* scale, int64_t n, int k, int row_first, int rows,
                                                            char* G, int64_t pitch) {
  const float f = scale ? *scale : 1.f;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int at = entries[i];
    if (at >= row_first && at - row_first < rows) store_out<T>(G, (int64_t)(at - row_first) * pitch + i / k, values[i] * f);
  }
}

}  // namespace gensor

namespace {

gensor_status check_teacher(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, int32_t k) {
  const gensor_status st = check_xent(dtype, T, V, D);
  if (st != GENSOR_OK) return st;
  return k < 1 || k > GENSOR_TEACHER_MAX ? GENSOR_ERR_INVALID_ARG : GENSOR_OK;
}

template <typename F>
hipError_t by_type(gensor_dtype dtype, F&& f) {
  if (dtype == GENSOR_F32) return f(f32_t{});
  return dtype == GENSOR_F16 ? f(f16_t{}) : f(bf16_t{});
}

TeacherArgs teacher_args(int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx, const void* W, int64_t ldw, float scale, int32_t k, const int64_t* index,
                         const float* teacher, int32_t normalize) {
  TeacherArgs a;
  std::memset(&a, 0, sizeof(a));
  a.X = (const char*)X; a.W = (const char*)W;
  a.ldx = ldx; a.ldw = ldw;
  a.index = index; a.teacher = teacher;
  a.T = (int32_t)T; a.V = (int32_t)V; a.D = (int32_t)D; a.k = k; a.normalize = normalize;
  a.scale = scale;
  return a;
}

bool whole_vectors(gensor_dtype dtype, int64_t D, const void* X, int64_t ldx, const void* W, int64_t ldw) {
  const int epc = 16 / size_of(dtype);
  return D % epc == 0 && ldx % epc == 0 && ldw % epc == 0 && aligned(X, 16) && aligned(W, 16);
}

unsigned token_blocks(int64_t T) { return (unsigned)std::min<int64_t>(T, 1 << 20); }

size_t teacher_room(int64_t T, int32_t k) { return round_up((size_t)T * 4 + (size_t)T * k * 8, 256); }

}  // namespace

extern "C" size_t gensor_distill_workspace_bytes(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, int32_t k, int32_t backward) {
  size_t bytes = 0;
  guarded([&]() -> gensor_status {
    if (check_teacher(dtype, T, V, D, k) != GENSOR_OK) return GENSOR_OK;
    bytes = backward ? teacher_room(T, k) + gensor_xent_workspace_bytes(dtype, T, V, D, 1) : round_up((size_t)T * 4, 256) + score_bytes(dtype, T, V, D, 0);
    return GENSOR_OK;
  });
  return bytes;
}

extern "C" gensor_status gensor_distill_forward(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx, const void* W, int64_t ldw, float scale,
                                                int32_t k, const int64_t* index, const float* teacher, int32_t normalize, float* loss, float* lse, void* workspace,
                                                size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> gensor_status {
  gensor_status st = check_teacher(dtype, T, V, D, k);
  if (st != GENSOR_OK) return st;
  if (!X || !W || ldx < D || ldw < D || !valid_scale(scale) || !index || !aligned(index, 8) || !teacher || (normalize != 0 && normalize != 1) || (!loss && !lse))
    return GENSOR_ERR_INVALID_ARG;
  const size_t head = round_up((size_t)T * 4, 256), room = usable_room(workspace, workspace_bytes);
  if (room < head) return GENSOR_ERR_WORKSPACE;
  float* sums = lse ? lse : (float*)workspace;
  hipStream_t s = (hipStream_t)hip_stream;
  const ScoreOutputs out = {nullptr, sums, nullptr, 0, nullptr, nullptr};
  st = run_scores(dtype, T, V, D, X, ldx, W, ldw, scale, nullptr, 0, out, (char*)workspace + head, room - head, s);
  if (st != GENSOR_OK || !loss) return st;
  TeacherArgs a = teacher_args(T, V, D, X, ldx, W, ldw, scale, k, index, teacher, normalize);
  a.lse = sums;
  a.loss = loss;
  const bool vec = whole_vectors(dtype, D, X, ldx, W, ldw);
  return launched(by_type(dtype, [&](auto type) {
    typedef decltype(type) E;
    if (vec) hipLaunchKernelGGL((teacher_loss_kernel<E, true>), dim3(token_blocks(T)), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((teacher_loss_kernel<E, false>), dim3(token_blocks(T)), dim3(256), 0, s, a);
    return hipGetLastError();
  }));
  });
}

extern "C" gensor_status gensor_distill_backward(gensor_dtype dtype, int64_t T, int64_t V, int64_t D, const void* X, int64_t ldx, const void* W, int64_t ldw, float scale,
                                                 int32_t k, const int64_t* index, const float* teacher, int32_t normalize, const float* lse, const float* dloss,
                                                 void* dX, int64_t lddx, void* dW, int64_t lddw, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> gensor_status {
  const gensor_status st = check_teacher(dtype, T, V, D, k);
  if (st != GENSOR_OK) return st;
  if (!X || !W || ldx < D || ldw < D || !valid_scale(scale) || !index || !aligned(index, 8) || !teacher || (normalize != 0 && normalize != 1)) return GENSOR_ERR_INVALID_ARG;
  if (!lse || !dloss || (!dX && !dW) || (dX && lddx < D) || (dW && lddw < D)) return GENSOR_ERR_INVALID_ARG;
  const size_t head = teacher_room(T, k), room = usable_room(workspace, workspace_bytes);
  if (room < head) return GENSOR_ERR_WORKSPACE;
  TeacherArgs a = teacher_args(T, V, D, X, ldx, W, ldw, scale, k, index, teacher, normalize);
  a.lse = lse;
  a.dloss = dloss;
  a.weights = (float*)workspace;
  a.entries = (int32_t*)(a.weights + T);
  a.values = (float*)(a.entries + T * k);
  const bool vec = whole_vectors(dtype, D, X, ldx, W, ldw);
  VocabularyLoss loss;
  loss.prepare = [&](float* scales, hipStream_t s) {
    const hipError_t e = by_type(dtype, [&](auto type) {
      typedef decltype(type) E;
      if (vec) hipLaunchKernelGGL((teacher_weights_kernel<E, true>), dim3(token_blocks(T)), dim3(256), 0, s, a);
      else hipLaunchKernelGGL((teacher_weights_kernel<E, false>), dim3(token_blocks(T)), dim3(256), 0, s, a);
      return hipGetLastError();
    });
    if (e != hipSuccess || !scales) return e;
    hipLaunchKernelGGL(teacher_scale_kernel, dim3(1), dim3(1024), 0, s, a.weights, (int)T, scales);
    return hipGetLastError();
  };
  loss.piece = [&](FusedArgs& f, const FusedDesc& tile, hipStream_t s) {
    f.alpha = scale;
    f.lse = lse;
    f.dloss = a.weights;
    const hipError_t e = g_lm_ends[&tile - g_fused].teach(f, s);
    if (e != hipSuccess) return e;
    const int64_t n = T * k;
    return by_type(dtype, [&](auto type) {
      hipLaunchKernelGGL((teacher_place_kernel<decltype(type)>), dim3((unsigned)std::min<int64_t>((n + 255) / 256, 1 << 20)), dim3(256), 0, s, a.entries, a.values, f.scale, n,
                         (int)k, f.row_first, f.M, (char*)f.C, f.ldc);
      return hipGetLastError();
    });
  };
  return vocabulary_gradient(dtype, T, V, D, X, ldx, W, ldw, loss, dX, lddx, dW, lddw, (char*)workspace + head, room - head, (hipStream_t)hip_stream);
  });
}
