// Products whose result is consumed where it is produced: what the contraction kernel's workgroups do with their tile in
// place of storing alpha * A * B (the F of contraction_kernel), and how they find their rows where the products are grouped.
//
//   END_LINEAR  C = act(alpha A B + bias) + residual, and the values before act kept; or C = (alpha A B) * act'(preact)
//   END_LSE     rows are vocabulary entries, columns tokens: each wave reduces its rows' logits to a maximum and a sum of
//               exponentials per token; nothing else is stored
//   END_PROB    the same product again: C = scale * dloss[token] * (exp(logit - lse[token]) - (row == target[token]))
//
//   MOVE_NONE   one product
//   MOVE_ROWS   group g owns rows [offsets[g], offsets[g+1]) of A and C and has its own B (and bias)
//   MOVE_DEPTH  group g owns k rows [offsets[g], offsets[g+1]) of both operands and has its own C
//
// Activations.  gelu is the tanh form, 0.5 z (1 + tanh(u)) with u = sqrt(2/pi) (z + 0.044715 z^3).  Since
// 0.5 (1 + tanh(u)) = sigmoid(2u), gelu and silu are both z * sigmoid(z (c1 + c2 z^2)), one exponential and one reciprocal,
// without the difference 1 + tanh that loses the negative side's digits.
#pragma once
#include "gemm_kernel.hpp"

namespace gensor {

enum { END_LINEAR = 0, END_LSE = 1, END_PROB = 2 };
enum { MOVE_NONE = PLACE_ALL, MOVE_ROWS = PLACE_ROWS, MOVE_DEPTH = PLACE_DEPTH };
enum { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };       // gensor_act

struct FusedArgs : KernelArgs {
  int32_t store_m, store_n;        // rows and columns of C that exist (loads go by M and N)
  // END_LINEAR
  int32_t act, grad;               // grad: C = (alpha A B) * act'(preact)
  const void* bias;                // of the input type, or null
  void* preact;                    // of C's type: written (read if grad), or null
  const void* residual;            // of C's type, or fp32 (residual_f32), or null
  int64_t ld_preact, ld_residual;
  int32_t residual_f32;
  const float* scale;              // one more factor of alpha, on the device, or null
  // groups
  const int32_t* offsets;          // groups + 1 of them; any values: what they name is cut to the `rows` there are
  int32_t groups, rows;
  int32_t tile_first;              // MOVE_ROWS: the tile of workgroup 0 (of a call's further launches)
  // END_LSE and END_PROB; a column is a token
  const int64_t* targets;
  int64_t ignore;
  const float* lse;
  const float* dloss;
  float* part_max;                 // [slab of C::WM rows][tokens]
  float* part_sum;
  float* at_target;                // the logit of the token's target
  int32_t tokens, row_first, vocab;        // row_first: vocabulary entry of row 0
};

// ---------------------------------------------------------------- activations
struct ActForm {
  float k1, k2, c1, c2;            // k = -log2(e) c
  __device__ explicit ActForm(int act) {
    constexpr float log2e = 1.44269504088896340736f;
    c1 = act == ACT_GELU ? 1.59576912160573071176f : 1.f;              // 2 sqrt(2 / pi)
    c2 = act == ACT_GELU ? 1.59576912160573071176f * 0.044715f : 0.f;
    k1 = -log2e * c1;
    k2 = -log2e * c2;
  }
  // (the square is held finite: 0 * inf would be NaN in silu's c2 z^2)
  __device__ float sigmoid(float z, float& q) const {
    q = fminf(z * z, 1e30f);
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * fmaf(k2, q, k1)));
  }
  __device__ float value(float z) const {
    float q;
    return z * sigmoid(z, q);
  }
  __device__ float slope(float z) const {
    float q;
    const float s = sigmoid(z, q);
    return fmaf(z * s * (1.f - s), fmaf(3.f * c2, q, c1), s);
  }
};

template <typename T> __device__ inline float from_bits(uint32_t u);
template <> __device__ inline float from_bits<f32_t>(uint32_t u) { return as_f32(u); }
template <> __device__ inline float from_bits<bf16_t>(uint32_t u) { return as_f32(u << 16); }
template <> __device__ inline float from_bits<f16_t>(uint32_t u) { return (float)__builtin_bit_cast(_Float16, (uint16_t)u); }
template <typename T> __device__ inline float from_pair(uint32_t u, int half);
template <> __device__ inline float from_pair<bf16_t>(uint32_t u, int half) { return as_f32(half ? u & 0xffff0000u : u << 16); }
template <> __device__ inline float from_pair<f16_t>(uint32_t u, int half) { return from_bits<f16_t>(half ? u >> 16 : u & 0xffffu); }

// ---------------------------------------------------------------- sums of exponentials
// sum = sum of exp(z - reference) with the maximum as the reference, or 0 where it is infinite (inf - inf): lse = reference + log(sum)
__device__ inline float lse_reference(float top) { return fabsf(top) == INFINITY ? 0.f : top; }
// ... joined with another part's.  (A part without terms has the maximum -inf and the sum 0: its factor must be no infinity.)
__device__ inline void join_sums(float& top, float& sum, float top2, float sum2) {
  constexpr float log2e = 1.44269504088896340736f;
  const float both = fmaxf(top, top2), r = lse_reference(both);
  const float f1 = fabsf(top) == INFINITY ? 1.f : __builtin_amdgcn_exp2f(log2e * (top - r));
  const float f2 = fabsf(top2) == INFINITY ? 1.f : __builtin_amdgcn_exp2f(log2e * (top2 - r));
  sum = sum * f1 + sum2 * f2;
  top = both;
}

// ---------------------------------------------------------------- groups
// Rows of group g: the offsets are device memory that the host never sees, so whatever they hold is cut to the rows there are.
__device__ inline void group_rows(const FusedArgs& a, int g, int& first, int& count) {
  first = min(max(a.offsets[g], 0), a.rows);
  count = min(max(a.offsets[g + 1], first), a.rows) - first;
}

// ---------------------------------------------------------------- the ends
template <int END, int MOVE>
struct Fused {
  typedef FusedArgs Args;
  static constexpr int MOVES = MOVE;
  static constexpr bool OWN_END = true;
  static constexpr bool STAYS = END == END_LSE, DUAL = false;
  // The rows of the first 64 groups, one a lane.
  static __device__ __attribute__((always_inline)) GroupRows own_group(const FusedArgs& a) {
    GroupRows r{0, -1};
    const int lane = threadIdx.x & 63;
    if (lane < a.groups) group_rows(a, lane, r.first, r.count);
    return r;
  }

  // Tile `id` of a launch; false: there is none.  The launch numbers as many as the row counts could need, ceil(rows / BM) of each group at
  // worst; every wave counts the tiles there are by itself (64 groups at a time, one a lane), so nothing has to run before this
  // launch and the host never waits for the counts.
  template <typename C>
  static __device__ __attribute__((always_inline)) bool place(const FusedArgs& a, int id, const GroupRows& own, GroupPlace& w) {
    const int lane = threadIdx.x & 63;
    if constexpr (MOVE == MOVE_DEPTH) {
      // The tiles of the group with the most rows start first, then the next one's: a tile's time is its group's rows, and a long
      // one started last would run alone.  Each group's tiles are dealt over all XCDs in contiguous ranges.  (Of more than 64
      // groups the order is kept among 64 at a time.)
      const int per = a.tiles_m * a.tiles_n;
      const int turn = id / per, g0 = turn & ~63;
      int first, count = own.count;
      if (g0 > 0) {
        count = -1;
        if (g0 + lane < a.groups) group_rows(a, g0 + lane, first, count);
      }
      int before = 0;
#pragma unroll 8
      for (int i = 0; i < 64; ++i) {
        const int other = __builtin_amdgcn_readlane(count, i);
        before += other > count || (other == count && i < lane);
      }
      w.group = g0 + __builtin_ctzll(__ballot(before == (turn & 63)));
      tile_of(a, xcd_contiguous(id - turn * per, per), w.tile_m, w.tile_n);
      group_rows(a, w.group, w.first, w.count);
      if (w.count > 0) return true;
      // nothing to add up: zeros
      typedef typename C::OutT OutT;
      char* c = (char*)a.C + (int64_t)w.group * a.strideC * ElemSize<OutT>::value;
      const int m0 = w.tile_m * C::BM, n0 = w.tile_n * C::BN;
      const int rows = min(C::BM, a.store_m - m0), cols = min(C::BN, a.store_n - n0);
      for (int i = threadIdx.x; i < rows * C::BN; i += C::THREADS) {
        const int r = i / C::BN, k = i % C::BN;
        if (k < cols) store_out<OutT>(c, (int64_t)(m0 + r) * a.ldc + n0 + k, 0.f);
      }
      return false;
    } else {
      auto rows_at = [&](int g0) {
        GroupRows r = own;
        if (g0 > 0) {
          r.count = 0;
          if (g0 + lane < a.groups) group_rows(a, g0 + lane, r.first, r.count);
        }
        return r;
      };
      auto tiles_at = [&](int g0) { return (max(rows_at(g0).count, 0) + C::BM - 1) / C::BM; };
      auto running = [&](int x) {                    // inclusive sum over the lanes
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
          const int y = __shfl_up(x, d, 64);
          if (lane >= d) x += y;
        }
        return x;
      };
      int total = 0, mine = 0;
      for (int g0 = 0; g0 < a.groups; g0 += 64) {
        mine = running(tiles_at(g0));
        total += __builtin_amdgcn_readlane(mine, 63);
      }
      total *= a.tiles_n;
      id += a.tile_first;
      if (id >= total) return false;
      const int t = xcd_contiguous(id, total);
      int before = 0;                                // tile rows of the groups before this chunk of them
      for (int g0 = 0; g0 < a.groups; g0 += 64) {
        if (a.groups > 64) mine = running(tiles_at(g0));
        const uint64_t beyond = __ballot((before + mine) * a.tiles_n > t);
        if (beyond != 0) {
          const int at = __builtin_ctzll(beyond);
          const int end = __builtin_amdgcn_readlane(mine, at);
          const int start = at > 0 ? __builtin_amdgcn_readlane(mine, at - 1) : 0;
          w.group = g0 + at;
          const GroupRows r = rows_at(g0);
          w.first = __builtin_amdgcn_readlane(r.first, at);
          w.count = __builtin_amdgcn_readlane(r.count, at);
          // the tiles of a group: panels of tile rows, walked column by column
          const int tile_rows = end - start, panel = min(a.panel, tile_rows), inside = t - (before + start) * a.tiles_n;
          const int pi = inside / (panel * a.tiles_n), rows_here = min(panel, tile_rows - pi * panel), q = inside - pi * panel * a.tiles_n;
          w.tile_m = pi * panel + q % rows_here;
          w.tile_n = q / rows_here;
          return true;
        }
        before += __builtin_amdgcn_readlane(mine, 63);
      }
      return false;
    }
  }

  // Reads lines that the tile's epilogue will read (two a thread), so that they lie in the L2 by then: 8192 x 3072 x 768, 16-bit, 42 us alone, with a
  // residual of 50 MB that is first asked for in the epilogue 63, so 57.  p.lane: the thread.
  template <typename C>
  static __device__ __attribute__((always_inline)) void touch(const FusedArgs& a, const TilePlace& p, uint32_t (&value)[2]) {
    if constexpr (END == END_LINEAR) {
      if (!a.residual && !a.grad) return;
      const EndPlace e = end_place<C>(a, p);
      const int size = a.residual && a.residual_f32 ? 4 : ElemSize<typename C::OutT>::value;
      const int64_t ld = a.residual ? a.ld_residual : a.ld_preact;
      const char* base = (const char*)(a.residual ? a.residual : a.preact) + (e.row0 * ld + p.n0) * size;
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, e.records(ld, size), 0x00020000u);
      const int per_row = (C::BN * size + 255) / 256;                  // threads a row; two lines each
      for (int at = p.lane; at < C::BM * per_row; at += C::THREADS) {
        const uint32_t off = (uint32_t)(at / per_row) * (uint32_t)(ld * size) + (uint32_t)(at % per_row) * 256u;
        value[0] = __builtin_amdgcn_raw_buffer_load_b32(r, off & ~3u, 0, 0);
        value[1] = __builtin_amdgcn_raw_buffer_load_b32(r, (off + 128u) & ~3u, 0, 0);
      }
    }
  }

  // Where the tile lies in C (and in what is read and kept beside it): its first row, and its rows and columns that exist.
  struct EndPlace {
    int64_t row0;
    int rows, cols, group;
    __device__ uint32_t records(int64_t ld, int size) const {
      const int64_t bytes = ((int64_t)(rows - 1) * ld + cols) * size;
      return bytes <= 0 ? 0u : bytes > 0x7fffffffll ? 0x7fffffffu : (uint32_t)bytes;
    }
  };
  template <typename C>
  static __device__ __attribute__((always_inline)) EndPlace end_place(const FusedArgs& a, const TilePlace& p) {
    return {(MOVE == MOVE_ROWS ? p.first : 0) + (int64_t)p.m0, min(C::BM, (MOVE == MOVE_ROWS ? p.count : a.store_m) - p.m0), min(C::BN, a.store_n - p.n0), p.group};
  }

  // before_stores: called where everything is computed and only stores follow (END_LSE)
  template <typename C, typename Acc, typename Hook>
  static __device__ __attribute__((always_inline)) void finish(const FusedArgs& a, Acc (&acc)[C::MBLK][C::NBLK], const TilePlace& p, Hook&& before_stores) {
    if constexpr (END == END_LSE) finish_lse<C>(a, acc, p, before_stores);
    else if constexpr (END == END_PROB) finish_prob<C>(a, acc, p);
    else finish_linear<C, true>(a, acc, p);
  }

  // Row of element v of a block, less the lane group's part (4 rows apart)
  template <typename C> static constexpr __device__ int row_of(int v) { return C::MB == 32 ? 8 * (v / 4) + v % 4 : v; }

  // ---- C = act(alpha A B + bias) + residual, or (alpha A B) * act'(preact); FULL = false: C = acc as it is.
  // Bound by what it moves beside C: the values kept or read again, and the residual.  An element access moves two bytes a
  // lane of 16-bit types, so where rows allow it (`paired`) pairs of rows of a column are traded with the neighbour lane for
  // pairs of columns of a row, as the plain epilogue does: the exchange is its own inverse, so what is read goes the
  // same way backwards.  (Four columns a lane, in half as many stores, were 3 us slower on 8192 x 3072 x 768: 41.3 -> 44.4.)
  // What is read is requested as far ahead as 32 registers hold: a load's wait counts the stores before it, too.
  // 8192 x 3072 x 768, us, on 16-bit types: nothing 42 (0.92 PFLOP/s), gelu 47, gelu with Z kept 57 (118 MB, 2.1 TB/s), a residual 57, the gradient through
  // gelu 62.  The products of all units and their stores take turns (two rounds of tiles in step), so the times add up: 28 of
  // products, 10 for each 50 MB moved, 5 for gelu's two transcendental operations a value.
  template <typename C, bool FULL, typename Acc>
  static __device__ __attribute__((always_inline)) void finish_linear(const FusedArgs& a, Acc (&acc)[C::MBLK][C::NBLK], const TilePlace& p) {
    typedef typename C::OutT OutT;
    constexpr int OS = ElemSize<OutT>::value, ES = C::ES, MB = C::MB, NACC = MB * MB / 64;
    constexpr uint32_t FLAGS = 0x00020000u, OOB = 0x80000000u;
    const int lane = p.lane, frow = lane % MB, fgrp = lane / MB;
    const EndPlace e = end_place<C>(a, p);
    const int cols_valid = e.cols;
    char* c_base = (char*)a.C + ((MOVE == MOVE_DEPTH ? (int64_t)e.group * a.strideC : 0) + e.row0 * a.ldc + p.n0) * OS;
    const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc((void*)c_base, 0, e.records(a.ldc, OS), FLAGS);
    const uint32_t pitch = (uint32_t)a.ldc * OS;
    const bool has_z = FULL && a.preact != nullptr, has_r = FULL && a.residual != nullptr;
    const int xs = has_r && a.residual_f32 ? 4 : OS;                   // size of what is read
    const bool reads = has_r || (has_z && a.grad);
    const char* x_base = has_r ? (const char*)a.residual : (const char*)a.preact;
    const int64_t x_ld = has_r ? a.ld_residual : a.ld_preact;
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)(reads ? x_base + (e.row0 * x_ld + p.n0) * xs : c_base), 0,
                                                                        reads ? e.records(x_ld, xs) : 0u, FLAGS);
    const uint32_t x_pitch = (uint32_t)x_ld * xs;
    const bool keeps = has_z && !a.grad;
    const __amdgpu_buffer_rsrc_t rz = __builtin_amdgcn_make_buffer_rsrc((void*)(keeps ? (char*)a.preact + (e.row0 * a.ld_preact + p.n0) * OS : c_base), 0,
                                                                        keeps ? e.records(a.ld_preact, OS) : 0u, FLAGS);
    const uint32_t z_pitch = (uint32_t)a.ld_preact * OS;
    const float alpha = FULL ? a.alpha * (a.scale ? *a.scale : 1.f) : 1.f;
    const int act = FULL ? a.act : ACT_NONE;
    const bool grad = FULL && a.grad;
    const ActForm form(act);

    // ---- bias: one value a lane and block column
    float bias[C::NBLK];
#pragma unroll
    for (int bj = 0; bj < C::NBLK; ++bj) {
      const int col = p.n0 + p.col + bj * MB + frow;
      bias[bj] = FULL && a.bias && col < a.store_n ? to_float<typename C::T>(a.bias, (MOVE == MOVE_ROWS ? (int64_t)e.group * a.N : 0) + col) : 0.f;
    }
    // the values of a block, x what was read for it; z: the values before the activation
    auto compute = [&](int bi, int bj, const float* x, float* z, float* y) {
#pragma unroll
      for (int v = 0; v < NACC; ++v) z[v] = FULL ? fmaf(alpha, acc[bi][bj][v], bias[bj]) : acc[bi][bj][v];
      if (act == ACT_NONE) {
#pragma unroll
        for (int v = 0; v < NACC; ++v) y[v] = z[v];
      } else if (grad) {
        if (act == ACT_RELU) {
#pragma unroll
          for (int v = 0; v < NACC; ++v) y[v] = x[v] > 0.f ? z[v] : 0.f;
        } else {
#pragma unroll
          for (int v = 0; v < NACC; ++v) y[v] = z[v] * form.slope(x[v]);
        }
      } else if (act == ACT_RELU) {
#pragma unroll
        for (int v = 0; v < NACC; ++v) y[v] = z[v] < 0.f ? 0.f : z[v];
      } else {
#pragma unroll
        for (int v = 0; v < NACC; ++v) y[v] = form.value(z[v]);
      }
      if (has_r) {
#pragma unroll
        for (int v = 0; v < NACC; ++v) y[v] += x[v];
      }
    };
    constexpr bool HALF_LINES = C::WN % 64 != 0;
    constexpr int GB = (HALF_LINES ? 32 : 64) / MB;                    // blocks side by side that are stored together
    constexpr bool PAIRS = OS == 2 && GB >= 2 && C::NBLK % GB == 0;
    if (PAIRS && a.paired) {
      if constexpr (PAIRS) {
        const uint32_t pick = (lane & 1) ? 0x03020706u : 0x05040100u;
        auto trade = [&](uint32_t own) -> uint32_t {
          const uint32_t other = (uint32_t)__builtin_amdgcn_mov_dpp((int)own, 0xB1, 0xF, 0xF, true);      // quad_perm [1,0,3,2]
          return __builtin_amdgcn_perm(other, own, pick);
        };
        constexpr int RS = GB == 4 ? 4 : 2;                            // stores of a pair of rows of GB blocks
        // w[i]: block i's pairs of rows v, v + 1; swapped into the order of the stores, whose rows are row_at(i) further down
        auto swap_in = [&](uint32_t* w) {
          if constexpr (MB == 32) {
            const auto q = __builtin_amdgcn_permlane32_swap(w[0], w[1], false, false);
            w[0] = q[0]; w[1] = q[1];
          } else if constexpr (GB == 2) {
            const auto q = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
            w[0] = q[0]; w[1] = q[1];
          } else {
            const auto s = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
            const auto t = __builtin_amdgcn_permlane16_swap(w[2], w[3], false, false);
            const auto c = __builtin_amdgcn_permlane32_swap(s[0], t[0], false, false);
            const auto d = __builtin_amdgcn_permlane32_swap(s[1], t[1], false, false);
            w[0] = c[0]; w[1] = d[0]; w[2] = c[1]; w[3] = d[1];
          }
        };
        auto swap_out = [&](uint32_t* w) {
          if constexpr (MB == 32) {
            const auto q = __builtin_amdgcn_permlane32_swap(w[0], w[1], false, false);
            w[0] = q[0]; w[1] = q[1];
          } else if constexpr (GB == 2) {
            const auto q = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
            w[0] = q[0]; w[1] = q[1];
          } else {
            const auto c = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
            const auto d = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
            const auto s = __builtin_amdgcn_permlane16_swap(c[0], d[0], false, false);
            const auto t = __builtin_amdgcn_permlane16_swap(c[1], d[1], false, false);
            w[0] = s[0]; w[1] = s[1]; w[2] = t[0]; w[3] = t[1];
          }
        };
        constexpr int UNITS = C::MBLK * (C::NBLK / GB), HALVES = NACC / 2;
        constexpr int AHEAD = UNITS * HALVES * RS <= 32 ? UNITS : 32 / (HALVES * RS);
        uint32_t in[AHEAD][HALVES][RS];
        auto column = [&](int bj) { return p.col + bj * MB + (lane % (GB * MB) & ~1); };
        auto row = [&](int bi) { return p.row + bi * MB + (lane & 1) + (HALF_LINES ? 8 * (lane >> 5) : 0); };
        auto request = [&](int u, int set) {
          const int bi = u % C::MBLK, bj = u / C::MBLK * GB;
          const uint32_t at = column(bj) < cols_valid ? (uint32_t)(column(bj) * OS) + (uint32_t)row(bi) * x_pitch : OOB;
#pragma unroll
          for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int i = 0; i < RS; ++i) in[set][h][i] = __builtin_amdgcn_raw_buffer_load_b32(rx, at + (uint32_t)(row_of<C>(2 * h) + 4 * i) * x_pitch, 0, 0);
        };
        if (reads) {
#pragma unroll
          for (int u = 0; u < AHEAD; ++u) request(u, u);
        }
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
          const int bi = u % C::MBLK, bj = u / C::MBLK * GB;
          float x[GB][NACC], z[GB][NACC], y[GB][NACC];
          if (reads) {
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
              uint32_t w[RS];
#pragma unroll
              for (int i = 0; i < RS; ++i) w[i] = in[u % AHEAD][h][i];
              swap_out(w);
#pragma unroll
              for (int g = 0; g < GB; ++g) {
                const uint32_t t = trade(w[g]);
                if constexpr (OS == 2) {
                  x[g][2 * h] = from_pair<OutT>(t, 0);
                  x[g][2 * h + 1] = from_pair<OutT>(t, 1);
                }
              }
            }
          }
          if (reads && u + AHEAD < UNITS) request(u + AHEAD, u % AHEAD);
#pragma unroll
          for (int g = 0; g < GB; ++g) compute(bi, bj + g, x[g], z[g], y[g]);
          auto put = [&](const float (&val)[GB][NACC], const __amdgpu_buffer_rsrc_t& r, uint32_t row_pitch) {
            const uint32_t at = column(bj) < cols_valid ? (uint32_t)(column(bj) * OS) + (uint32_t)row(bi) * row_pitch : OOB;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
              uint32_t w[RS];
#pragma unroll
              for (int g = 0; g < GB; ++g) w[g] = trade(pack_out<OutT>(val[g][2 * h], val[g][2 * h + 1]));
              swap_in(w);
#pragma unroll
              for (int i = 0; i < RS; ++i) {
                const uint32_t off = at + (uint32_t)(row_of<C>(2 * h) + 4 * i) * row_pitch;
                if (a.through) __builtin_amdgcn_raw_buffer_store_b32(w[i], r, off, 0, 16);
                else __builtin_amdgcn_raw_buffer_store_b32(w[i], r, off, 0, 0);
              }
            }
          };
          if (keeps) put(z, rz, z_pitch);
          put(y, rc, pitch);
        }
      }
      return;
    }
    // ---- element accesses
    constexpr int BLOCKS = C::MBLK * C::NBLK;
    constexpr int AHEAD = BLOCKS * NACC <= 32 ? BLOCKS : 32 / NACC;
    uint32_t in[AHEAD][NACC];
    auto column = [&](int bj) { return p.col + bj * MB + frow; };
    auto row = [&](int bi) { return p.row + bi * MB + 4 * fgrp; };
    auto request = [&](int b, int set) {
      const int bi = b % C::MBLK, bj = b / C::MBLK;
      const uint32_t at = column(bj) < cols_valid ? (uint32_t)(column(bj) * xs) + (uint32_t)row(bi) * x_pitch : OOB;
      if (xs == 4) {
#pragma unroll
        for (int v = 0; v < NACC; ++v) in[set][v] = __builtin_amdgcn_raw_buffer_load_b32(rx, at + (uint32_t)row_of<C>(v) * x_pitch, 0, 0);
      } else {
#pragma unroll
        for (int v = 0; v < NACC; ++v) in[set][v] = __builtin_amdgcn_raw_buffer_load_b16(rx, at + (uint32_t)row_of<C>(v) * x_pitch, 0, 0);
      }
    };
    if (reads) {
#pragma unroll
      for (int b = 0; b < AHEAD; ++b) request(b, b);
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const int bi = b % C::MBLK, bj = b / C::MBLK;
      float x[NACC], z[NACC], y[NACC];
      if (reads) {
#pragma unroll
        for (int v = 0; v < NACC; ++v) x[v] = OS == 4 || xs == 4 ? as_f32(in[b % AHEAD][v]) : from_bits<OutT>(in[b % AHEAD][v]);
      }
      if (reads && b + AHEAD < BLOCKS) request(b + AHEAD, b % AHEAD);
      compute(bi, bj, x, z, y);
      auto put = [&](const float* val, const __amdgpu_buffer_rsrc_t& r, uint32_t row_pitch, auto policy_tag) {
        constexpr int policy = decltype(policy_tag)::value;
        const uint32_t at = column(bj) < cols_valid ? (uint32_t)(column(bj) * OS) + (uint32_t)row(bi) * row_pitch : OOB;
#pragma unroll
        for (int v = 0; v < NACC; ++v) {
          const uint32_t off = at + (uint32_t)row_of<C>(v) * row_pitch;
          if constexpr (OS == 4) {
            __builtin_amdgcn_raw_buffer_store_b32(as_u32(val[v]), r, off, 0, policy);
          } else {
            uint16_t bits;
            store_out<OutT>(&bits, 0, val[v]);
            __builtin_amdgcn_raw_buffer_store_b16(bits, r, off, 0, policy);
          }
        }
      };
      if (a.through) {
        if (keeps) put(z, rz, z_pitch, std::integral_constant<int, 16>{});
        put(y, rc, pitch, std::integral_constant<int, 16>{});
      } else {
        if (keeps) put(z, rz, z_pitch, std::integral_constant<int, 0>{});
        put(y, rc, pitch, std::integral_constant<int, 0>{});
      }
    }
  }

  // ---- the logits of a wave's rows (vocabulary entries) reduced for each column (token).  A lane's registers are rows of one
  // column, so the reduction stays inside the lane but for the two or four lane groups of a block at the end: with the tokens
  // as rows it would cross 32 lanes for every row.  Bound by the products; then by the vector unit, three operations and an exponential a
  // logit, 3 us of a tile's 22.  8192 tokens, 50257 entries, 768 wide, f16: 560 to 600 us with the join's 8, 1.05 to 1.13 PFLOP/s (matrix units busy 54 % of the
  // cycles, 0.97 GB read), where the product that stores its logits takes 645.
  template <typename C, typename Acc, typename Hook>
  static __device__ __attribute__((always_inline)) void finish_lse(const FusedArgs& a, Acc (&acc)[C::MBLK][C::NBLK], const TilePlace& p, Hook&& before_stores) {
    constexpr int MB = C::MB, NACC = MB * MB / 64;
    constexpr float log2e = 1.44269504088896340736f;
    const int lane = p.lane, frow = lane % MB, fgrp = lane / MB;
    const int first = p.m0 + p.row;                                  // the wave's first row
    const int rows = min(C::WM, a.store_m - first);
    const int slab = first / C::WM;
    float tops[C::NBLK], sums[C::NBLK], at_target[C::NBLK];
    bool hit[C::NBLK];
#pragma unroll
    for (int bj = 0; bj < C::NBLK; ++bj) {
      const int token = p.n0 + p.col + bj * MB + frow;
      const bool there = token < a.store_n;
      float top = -INFINITY;
      if (rows < C::WM) {
#pragma unroll
        for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
          for (int v = 0; v < NACC; ++v)
            if (bi * MB + row_of<C>(v) + 4 * fgrp >= rows) acc[bi][bj][v] = -INFINITY;
      }
#pragma unroll
      for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
        for (int v = 0; v < NACC; ++v) top = fmaxf(top, acc[bi][bj][v]);
      // exp(z - ref) in three operations: the product log2e * ref is rounded, which multiplies every term by the same factor 2^off; it is taken
      // out of the sum, so that the maximum's own term is 1.  (off is up to 2^-24 of the product.  Beyond 1e9, where it may exceed 64 and its power all
      // numbers: four operations.  A stretch of the vocabulary that is shut off with large negative logits comes here, too.  The column's own choice: a
      // token's bits do not depend on what its neighbours hold.)
      const float ref = lse_reference(top);
      const bool far = fabsf(ref) > 1e9f;
      const float base = far ? 0.f : -(log2e * ref), off = far ? 0.f : fmaf(log2e, ref, base);
      float sum = 0.f;
      if (__any(far)) {
#pragma unroll
        for (int bi = 0; bi < C::MBLK; ++bi) {
          float part = 0.f;
#pragma unroll
          for (int v = 0; v < NACC; ++v) part += __builtin_amdgcn_exp2f(far ? log2e * (acc[bi][bj][v] - ref) : fmaf(log2e, acc[bi][bj][v], base));
          sum += part;
        }
      } else {
#pragma unroll
        for (int bi = 0; bi < C::MBLK; ++bi) {
          float part = 0.f;
#pragma unroll
          for (int v = 0; v < NACC; ++v) part += __builtin_amdgcn_exp2f(fmaf(log2e, acc[bi][bj][v], base));
          sum += part;
        }
      }
      sum *= __builtin_amdgcn_exp2f(-off);
#pragma unroll
      for (int d = MB; d < 64; d *= 2) {
        const float t2 = __shfl_xor(top, d, 64), s2 = __shfl_xor(sum, d, 64);
        join_sums(top, sum, t2, s2);
      }
      tops[bj] = top;
      sums[bj] = sum;
      hit[bj] = false;
      at_target[bj] = 0.f;
      if (a.targets) {
        const int64_t target = there ? a.targets[token] : -1;
        const int64_t entry = (int64_t)first + a.row_first;
        const int at = target != a.ignore && target >= entry && target < entry + rows ? (int)(target - entry) - 4 * fgrp : -1;
        if (__any(at >= 0)) {
#pragma unroll
          for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
            for (int v = 0; v < NACC; ++v)
              if (at == bi * MB + row_of<C>(v)) {
                hit[bj] = true;
                at_target[bj] = acc[bi][bj][v];
              }
        }
      }
    }
    before_stores();
#pragma unroll
    for (int bj = 0; bj < C::NBLK; ++bj) {
      const int token = p.n0 + p.col + bj * MB + frow;
      if (token < a.store_n && fgrp == 0 && rows > 0) {
        a.part_max[(int64_t)slab * a.tokens + token] = tops[bj];
        a.part_sum[(int64_t)slab * a.tokens + token] = sums[bj];
      }
      if (hit[bj]) a.at_target[token] = at_target[bj];
    }
  }

  // exp(z - lse), base = -log2(e) lse.  For 16-bit results in two operations: base is rounded, up to an lse of 1024 by 2^-14, a factor within 2^-14
  // of one, where the results are rounded by 2^-11 and 2^-8 (below_lse takes care of what lies beyond).  In fp32 the exponent's
  // rounding (2^-24 of up to a hundred) is carried as a factor.
  template <typename C> static __device__ float probability(float z, float lse, float base) {
    constexpr float log2e = 1.44269504088896340736f;
    if constexpr (C::ES == 2) return __builtin_amdgcn_exp2f(fmaf(log2e, z, base));
    const float d = z - lse, t = log2e * d;
    const float r = fmaf(log2e, d, -t) + 1.92596299e-8f * d;           // (log2(e) - log2e)
    const float e = __builtin_amdgcn_exp2f(t);
    return d > -100.f ? fmaf(e, 0.69314718f * r, e) : e;                // (-inf: inf - inf)
  }
  // The `base` of a column's probabilities.  16-bit types, an lse beyond 1024: the logits become their differences from it, one operation more, and base 0.
  // (Only of the waves that have such a token, and the token's own choice: with the rounded product a probability of one could be up to 2^64 at an lse of
  // 1e9, and infinite from some 3e9 on.)
  template <typename C, typename Acc>
  static __device__ __attribute__((always_inline)) float below_lse(Acc (&acc)[C::MBLK][C::NBLK], int bj, float lse, bool counts) {
    constexpr int NACC = C::MB * C::MB / 64;
    if constexpr (C::ES == 2) {
      const bool far = counts && fabsf(lse) > 1024.f;
      if (__any(far)) {
        const float off = far ? lse : 0.f;
#pragma unroll
        for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
          for (int v = 0; v < NACC; ++v) acc[bi][bj][v] -= off;
      }
      return far ? 0.f : -1.44269504088896340736f * lse;
    }
    return 0.f;
  }

  // ---- scale * dloss * (softmax - one at the target), in the input type, a product's operand next.  Columns beyond the tokens,
  // up to whole vectors (store_n), are written as zeros.  4096 tokens, 50257 entries, 768 wide, bf16: 340 to 360 us in two pieces,
  // 0.88 to 0.93 PFLOP/s.
  template <typename C, typename Acc>
  static __device__ __attribute__((always_inline)) void finish_prob(const FusedArgs& a, Acc (&acc)[C::MBLK][C::NBLK], const TilePlace& p) {
    constexpr int MB = C::MB, NACC = MB * MB / 64;
    const int lane = p.lane, frow = lane % MB, fgrp = lane / MB;
    const int first = p.m0 + p.row + a.row_first;
    const float scale = a.scale ? *a.scale : 1.f;
#pragma unroll
    for (int bj = 0; bj < C::NBLK; ++bj) {
      const int token = p.n0 + p.col + bj * MB + frow;
      const bool there = token < a.tokens;
      const int64_t target = there ? a.targets[token] : -1;
      const bool counts = there && target != a.ignore && target >= 0 && target < a.vocab;
      const float lse = counts ? a.lse[token] : INFINITY, base = below_lse<C>(acc, bj, lse, counts), g = counts ? a.dloss[token] * scale : 0.f;
      // (zero by choice, not by g = 0: the logits of a token that does not count may be infinite or NaN)
#pragma unroll
      for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
        for (int v = 0; v < NACC; ++v) acc[bi][bj][v] = counts ? g * probability<C>(acc[bi][bj][v], lse, base) : 0.f;
      const int at = counts && target >= first && target < (int64_t)first + C::WM ? (int)(target - first) - 4 * fgrp : -1;
      if (__any(at >= 0)) {
#pragma unroll
        for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
          for (int v = 0; v < NACC; ++v)
            if (at == bi * MB + row_of<C>(v)) acc[bi][bj][v] -= g;
      }
    }
    finish_linear<C, false>(a, acc, p);
  }
};

// One element of C from its product's sum, through the linear end.
template <typename T, typename OutT>
__device__ inline void finish_element(const FusedArgs& args, int m, int n, float sum) {
  const float alpha = args.alpha * (args.scale ? *args.scale : 1.f);
  const float z = fmaf(alpha, sum, args.bias ? to_float<T>(args.bias, n) : 0.f);
  const ActForm form(args.act);
  float y = z;
  if (args.preact && args.grad) {
    const float at = to_float<OutT>(args.preact, (int64_t)m * args.ld_preact + n);
    if (args.act == ACT_RELU) y = at > 0.f ? z : 0.f;
    else if (args.act != ACT_NONE) y = z * form.slope(at);
  } else {
    if (args.preact) store_out<OutT>(args.preact, (int64_t)m * args.ld_preact + n, z);
    if (args.act == ACT_RELU) y = z < 0.f ? 0.f : z;
    else if (args.act != ACT_NONE) y = form.value(z);
  }
  if (args.residual) {
    const int64_t i = (int64_t)m * args.ld_residual + n;
    y += args.residual_f32 ? to_float<f32_t>(args.residual, i) : to_float<OutT>(args.residual, i);
  }
  store_out<OutT>(args.C, (int64_t)m * args.ldc + n, y);
}

// A split tile: the sum of its slots, through the same end.  (The slots' order and the reasons for a second launch stand at
// split_reduce.)
template <typename T, typename OutT>
__global__ __launch_bounds__(256) void fused_split_reduce(const FusedArgs args, int bm, int bn, int wm, int wn, int mb) {
  const int threads = (bm / wm) * (bn / wn) * 64;
  const int groups = bm * bn / 4, blocks = groups >> 8;
  const int u = blockIdx.x / blocks, r = (blockIdx.x - u * blocks) * 256 + threadIdx.x;
  const int g = r / threads, tid = r - g * threads;
  const int lane = tid & 63, wave = tid >> 6, waves_n = bn / wn, nblk = wn / mb;
  const int per_block = mb == 32 ? 4 : 1;
  const int b = g / per_block, q = g - b * per_block;
  const int row = (wave / waves_n) * wm + (b / nblk) * mb + 8 * q + 4 * (lane / mb);
  const int col = (wave % waves_n) * wn + (b % nblk) * mb + lane % mb;
  const __amdgpu_buffer_rsrc_t slots = __builtin_amdgcn_make_buffer_rsrc((void*)((const f32x4*)args.partials + (int64_t)u * args.split * groups), 0,
                                                                        (uint32_t)(args.split * groups * 16), 0x00020000u);
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](auto n_tag) {
    constexpr int n = decltype(n_tag)::value;
    u32x4 v[n];
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = __builtin_amdgcn_raw_buffer_load_b128(slots, (uint32_t)((i * groups + r) * 16), 0, 2 /* nt */);
#pragma unroll
    for (int i = 0; i < n; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) sum[x] += as_f32(v[i][x]);
  };
  if (args.split <= 2) add(std::integral_constant<int, 2>{});
  else if (args.split <= 4) add(std::integral_constant<int, 4>{});
  else if (args.split <= 8) add(std::integral_constant<int, 8>{});
  else add(std::integral_constant<int, 16>{});
  int tile_m, tile_n;
  tile_of(args, args.whole + u, tile_m, tile_n);
  const int m = tile_m * bm + row, n = tile_n * bn + col;
  if (n >= args.store_n) return;
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (m + x < args.store_m) finish_element<T, OutT>(args, m + x, n, sum[x]);
}

}  // namespace gensor
