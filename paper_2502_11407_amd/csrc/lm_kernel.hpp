// Ends of the contraction kernel for a language model's gated layers, for the scores of a vocabulary and for learning from a teacher
// (the F of contraction_kernel):
//
//   Gated      C = act(G) * U of the two products G = alpha A B0 + b0 and U = alpha A B1 + b1, which may be kept
//   GatedGrad  of the gradient D = alpha A B of that C:  dG = D U act'(G),  dU = D act(G),  and C = act(G) U again
//   Score      rows are vocabulary entries, columns tokens: each wave reduces its rows' logits to a maximum, a sum of exponentials and their
//              sum weighted with the logits per token; where the largest entries are asked for, the maxima of sets of rows are left too, and the
//              logits themselves of those sets that may hold one
//   Teach      the same product again: C = scale * weight[token] * exp(logit - lse[token])
#pragma once
#include "fused_kernel.hpp"
#include "score_order.hpp"

namespace gensor {

// of a lambda that holds what it names by reference: called, these would lie in memory, a tile's descriptors among them
#define GENSOR_INLINE __attribute__((always_inline))

struct GatedArgs : KernelArgs {
  int32_t act;
  const void* bias;                // [2][N] of the input type, or null
  void* preact;                    // G, and U `far_preact` elements behind it: written, or null (GatedGrad: read)
  int64_t ld_preact, far_preact;
  void* dpreact;                   // GatedGrad: dG and dU
  int64_t ld_dpreact, far_dpreact;
};

struct ScoreArgs : KernelArgs {
  const int64_t* targets;
  int64_t ignore;
  int32_t tokens, row_first, vocab;        // row_first: vocabulary entry of row 0
  int32_t weighted;                        // the weighted sum is wanted
  int32_t slabs, sets;                     // of a token's row of `parts` and of `set_max` (0: the largest are not asked for)
  f32x4* parts;                            // [token][slab of C::WM rows]: maximum, sum, weighted sum
  float* set_max;                          // [token][set of rows]
  float* logits;                           // [token][set][rows of a set]: what is read of a token lies close together
  const float* bar;                        // logits of sets whose maximum is not above a token's are not needed, and not stored (NaN, or null: all are)
  float* at_target;
};

// Rows of a set: as many as one set's logits, 128 bytes a token, fill of a line, of a wave's tile
__host__ __device__ constexpr int score_set(int wm) { return wm < 32 ? wm : 32; }

// ---------------------------------------------------------------- 16-bit values of MFMA blocks in whole dwords
// A lane's registers are rows of one column, two bytes each in C.  Pairs of rows of a column are traded with the neighbour lane for pairs of
// columns of a row, and of GB blocks side by side the lane groups' parts are gathered, so that a store writes runs of 32 GB bytes (blocks of
// 16) or 64 GB (blocks of 32).  The exchange is its own inverse: what is read goes the same way backwards.  WIDTH: the columns of the wave's
// part.  A pair of rows of GB blocks takes RS accesses, 4 rows apart.
template <typename C, int WIDTH>
struct Paired {
  static constexpr int MB = C::MB, GB = WIDTH % 64 == 0 ? 64 / MB : WIDTH % 32 == 0 ? 32 / MB : 1, RS = GB;
  static __device__ uint32_t trade(uint32_t own) {
    const uint32_t other = (uint32_t)__builtin_amdgcn_mov_dpp((int)own, 0xB1, 0xF, 0xF, true);      // quad_perm [1,0,3,2]
    return __builtin_amdgcn_perm(other, own, (threadIdx.x & 1) ? 0x03020706u : 0x05040100u);
  }
  static __device__ void swap16(uint32_t& x, uint32_t& y) {
    const auto q = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    x = q[0]; y = q[1];
  }
  static __device__ void swap32(uint32_t& x, uint32_t& y) {
    const auto q = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    x = q[0]; y = q[1];
  }
  // w[i]: block i's pair of rows -> access i's
  static __device__ __attribute__((always_inline)) void gather(uint32_t (&w)[RS]) {
    if constexpr (GB == 2 && MB == 32) swap32(w[0], w[1]);
    else if constexpr (GB == 2) swap16(w[0], w[1]);
    else if constexpr (GB == 4) {
      swap16(w[0], w[1]);
      swap16(w[2], w[3]);
      swap32(w[0], w[2]);
      swap32(w[1], w[3]);
    }
  }
  static __device__ __attribute__((always_inline)) void scatter(uint32_t (&w)[RS]) {
    if constexpr (GB == 2 && MB == 32) swap32(w[0], w[1]);
    else if constexpr (GB == 2) swap16(w[0], w[1]);
    else if constexpr (GB == 4) {
      swap32(w[0], w[2]);
      swap32(w[1], w[3]);
      swap16(w[0], w[1]);
      swap16(w[2], w[3]);
    }
  }
  // first row (of the pair's row_of) and column of this lane's accesses
  static __device__ int row(int lane) { return (lane & 1) + (GB == 1 ? 4 * (lane / MB) : GB * MB == 32 ? 8 * (lane >> 5) : 0); }
  static __device__ int column(int lane) { return lane % (GB * MB) & ~1; }
};

template <typename C> static constexpr __device__ int block_row_of(int v) { return C::MB == 32 ? 8 * (v / 4) + v % 4 : v; }

// The descriptor of a matrix beside C, from the tile's first place to its last.  (Null: nothing is read and nothing written.)
__device__ __attribute__((always_inline)) inline __amdgpu_buffer_rsrc_t tile_matrix(const void* base, int64_t ld, int64_t row, int64_t col, int rows, int cols, int size) {
  const int64_t bytes = base ? ((int64_t)(rows - 1) * ld + cols) * size : 0;
  return __builtin_amdgcn_make_buffer_rsrc((void*)(base ? (const char*)base + (row * ld + col) * size : nullptr), 0,
                                           bytes <= 0 ? 0u : bytes > 0x7fffffffll ? 0x7fffffffu : (uint32_t)bytes, 0x00020000u);
}

// One wave's blocks of a matrix beside C: MBLK x BLOCKS of them, the first column at `col` of the tile.
template <typename C, int BLOCKS>
struct WaveBlocks {
  typedef typename C::OutT OutT;
  static constexpr int OS = ElemSize<OutT>::value, MB = C::MB, NACC = MB * MB / 64, WIDTH = BLOCKS * MB;
  typedef Paired<C, WIDTH> P;
  static constexpr int GB = OS == 2 ? P::GB : 1, RS = OS == 2 ? P::RS : 1, HALVES = NACC / 2;
  static constexpr uint32_t OOB = 0x80000000u;
  int row0, col0, cols, lane;

  // ---- pairs (16-bit types, rows of whole dwords): unit (bi, bj .. bj + GB - 1)
  __device__ __attribute__((always_inline)) uint32_t at_pair(uint32_t pitch, int bi, int bj) const {
    const int c = col0 + bj * MB + P::column(lane);
    return c < cols ? (uint32_t)(c * OS) + (uint32_t)(row0 + bi * MB + P::row(lane)) * pitch : OOB;
  }
  __device__ __attribute__((always_inline)) void request_pair(__amdgpu_buffer_rsrc_t r, uint32_t pitch, int bi, int bj, uint32_t (&in)[HALVES][RS]) const {
    const uint32_t at = at_pair(pitch, bi, bj);
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
#pragma unroll
      for (int i = 0; i < RS; ++i) in[h][i] = __builtin_amdgcn_raw_buffer_load_b32(r, at + (uint32_t)(block_row_of<C>(2 * h) + 4 * i) * pitch, 0, 0);
  }
  // rows 2h and 2h + 1 of the blocks
  __device__ __attribute__((always_inline)) void received_half(const uint32_t (&in)[RS], float (&x)[GB][2]) const {
    if constexpr (OS == 2) {
      uint32_t w[RS];
#pragma unroll
      for (int i = 0; i < RS; ++i) w[i] = in[i];
      P::scatter(w);
#pragma unroll
      for (int g = 0; g < GB; ++g) {
        const uint32_t t = P::trade(w[g]);
        x[g][0] = from_pair<OutT>(t, 0);
        x[g][1] = from_pair<OutT>(t, 1);
      }
    }
  }
  __device__ __attribute__((always_inline)) void store_half(__amdgpu_buffer_rsrc_t r, uint32_t pitch, uint32_t at, int h, const float (&val)[GB][2], bool through) const {
    if constexpr (OS == 2) {
      uint32_t w[RS];
#pragma unroll
      for (int g = 0; g < GB; ++g) w[g] = P::trade(pack_out<OutT>(val[g][0], val[g][1]));
      P::gather(w);
#pragma unroll
      for (int i = 0; i < RS; ++i) {
        const uint32_t off = at + (uint32_t)(block_row_of<C>(2 * h) + 4 * i) * pitch;
        if (through) __builtin_amdgcn_raw_buffer_store_b32(w[i], r, off, 0, 16);
        else __builtin_amdgcn_raw_buffer_store_b32(w[i], r, off, 0, 0);
      }
    }
  }
  // ---- single elements: block (bi, bj)
  __device__ __attribute__((always_inline)) uint32_t at_one(uint32_t pitch, int bi, int bj) const {
    const int c = col0 + bj * MB + lane % MB;
    return c < cols ? (uint32_t)(c * OS) + (uint32_t)(row0 + bi * MB + 4 * (lane / MB)) * pitch : OOB;
  }
  __device__ __attribute__((always_inline)) void request_one(__amdgpu_buffer_rsrc_t r, uint32_t pitch, int bi, int bj, uint32_t (&in)[NACC]) const {
    const uint32_t at = at_one(pitch, bi, bj);
#pragma unroll
    for (int v = 0; v < NACC; ++v) {
      if constexpr (OS == 4) in[v] = __builtin_amdgcn_raw_buffer_load_b32(r, at + (uint32_t)block_row_of<C>(v) * pitch, 0, 0);
      else in[v] = __builtin_amdgcn_raw_buffer_load_b16(r, at + (uint32_t)block_row_of<C>(v) * pitch, 0, 0);
    }
  }
  __device__ __attribute__((always_inline)) void received_one(const uint32_t (&in)[NACC], float (&x)[NACC]) const {
#pragma unroll
    for (int v = 0; v < NACC; ++v) x[v] = from_bits<OutT>(in[v]);
  }
  __device__ __attribute__((always_inline)) void store_one(__amdgpu_buffer_rsrc_t r, uint32_t pitch, int bi, int bj, const float (&val)[NACC], bool through) const {
    const uint32_t at = at_one(pitch, bi, bj);
#pragma unroll
    for (int v = 0; v < NACC; ++v) {
      const uint32_t off = at + (uint32_t)block_row_of<C>(v) * pitch;
      if constexpr (OS == 4) {
        if (through) __builtin_amdgcn_raw_buffer_store_b32(as_u32(val[v]), r, off, 0, 16);
        else __builtin_amdgcn_raw_buffer_store_b32(as_u32(val[v]), r, off, 0, 0);
      } else {
        uint16_t bits;
        store_out<OutT>(&bits, 0, val[v]);
        if (through) __builtin_amdgcn_raw_buffer_store_b16(bits, r, off, 0, 16);
        else __builtin_amdgcn_raw_buffer_store_b16(bits, r, off, 0, 0);
      }
    }
  }
};

// ---------------------------------------------------------------- the ends
// Both products of a place of C lie in the same lane (a wave's columns of the B tile are half of either matrix), so G, U and the result never leave the
// registers before they are stored.  Bound by the products and, with G and U kept, by storing three values where a product stores one: all units end a
// round of tiles together, so the times add up.  8192 x 768 -> 2 x 2048, us, 16-bit types: 46 to 50 (1.03 to 1.12 PFLOP/s), with G and U kept 55 to 61 (76 MB read,
// 101 written, matrix units busy 35 % of the cycles); 2048 x 2048 -> 2 x 5632 with gelu, 256x128 tiles, 84 to 92 (1.03 to 1.13 PFLOP/s, busy 48 %).
struct Gated {
  typedef GatedArgs Args;
  static constexpr int MOVES = PLACE_ALL;
  static constexpr bool OWN_END = true, STAYS = false, DUAL = true;
  template <typename C>
  static __device__ __attribute__((always_inline)) void touch(const Args&, const TilePlace&, uint32_t (&)[2]) {}

  template <typename C, typename Acc, typename Hook>
  static __device__ __attribute__((always_inline)) void finish(const Args& a, Acc (&acc)[C::MBLK][C::NBLK], const TilePlace& p, Hook&&) {
    constexpr int B2 = C::NBLK / 2, MB = C::MB, NACC = MB * MB / 64;
    typedef WaveBlocks<C, B2> W;
    const int rows = min(C::BM, a.M - p.m0), cols = min(C::BN / 2, a.N - p.n0);
    const W w{p.row, p.col / 2, cols, p.lane};
    const uint32_t pitch_c = (uint32_t)(a.ldc * W::OS), pitch_z = (uint32_t)(a.ld_preact * W::OS);
    const __amdgpu_buffer_rsrc_t c = tile_matrix(a.C, a.ldc, p.m0, p.n0, rows, cols, W::OS);
    const __amdgpu_buffer_rsrc_t g = tile_matrix(a.preact, a.ld_preact, p.m0, p.n0, rows, cols, W::OS);
    const __amdgpu_buffer_rsrc_t u = tile_matrix(a.preact ? (char*)a.preact + a.far_preact * W::OS : nullptr, a.ld_preact, p.m0, p.n0, rows, cols, W::OS);
    const bool keeps = a.preact != nullptr, through = a.through;
    const ActForm form(a.act);
    float bias[2][B2];
#pragma unroll
    for (int bj = 0; bj < B2; ++bj) {
      const int col = p.n0 + w.col0 + bj * MB + p.lane % MB;
      const bool there = a.bias && col < a.N;
      bias[0][bj] = there ? to_float<typename C::T>(a.bias, col) : 0.f;
      bias[1][bj] = there ? to_float<typename C::T>(a.bias, (int64_t)a.N + col) : 0.f;
    }
    // (every index is a constant: accumulators that are indexed in a loop would lie in memory)
    auto compute = [&](auto bi, auto bj, auto first, auto& zg, auto& zu, auto& y) GENSOR_INLINE {
      constexpr int N = sizeof(y) / sizeof(float);
#pragma unroll
      for (int v = 0; v < N; ++v) {
        zg[v] = fmaf(a.alpha, acc[bi][bj][first + v], bias[0][bj]);
        zu[v] = fmaf(a.alpha, acc[bi][bj + B2][first + v], bias[1][bj]);
      }
      if (a.act == ACT_NONE) {
#pragma unroll
        for (int v = 0; v < N; ++v) y[v] = zg[v] * zu[v];
      } else if (a.act == ACT_RELU) {
#pragma unroll
        for (int v = 0; v < N; ++v) y[v] = (zg[v] < 0.f ? 0.f : zg[v]) * zu[v];
      } else {
#pragma unroll
        for (int v = 0; v < N; ++v) y[v] = form.value(zg[v]) * zu[v];
      }
    };
    if (W::OS == 2 && a.paired) {
      static_for<B2 / W::GB * C::MBLK>([&](auto n) GENSOR_INLINE {
        constexpr std::integral_constant<int, n % C::MBLK> bi{};
        constexpr int bj = n / C::MBLK * W::GB;
        const uint32_t at_g = w.at_pair(pitch_z, bi, bj), at_u = w.at_pair(pitch_z, bi, bj), at_c = w.at_pair(pitch_c, bi, bj);
        static_for<W::HALVES>([&](auto h) GENSOR_INLINE {
          float zg[W::GB][2], zu[W::GB][2], y[W::GB][2];
          static_for<W::GB>([&](auto i) GENSOR_INLINE { compute(bi, std::integral_constant<int, bj + i>{}, std::integral_constant<int, 2 * h>{}, zg[i], zu[i], y[i]); });
          if (keeps) {
            w.store_half(g, pitch_z, at_g, h, zg, through);
            w.store_half(u, pitch_z, at_u, h, zu, through);
          }
          w.store_half(c, pitch_c, at_c, h, y, through);
        });
      });
      return;
    }
    static_for<B2 * C::MBLK>([&](auto n) GENSOR_INLINE {
      constexpr std::integral_constant<int, n % C::MBLK> bi{};
      constexpr std::integral_constant<int, n / C::MBLK> bj{};
      float zg[NACC], zu[NACC], y[NACC];
      compute(bi, bj, std::integral_constant<int, 0>{}, zg, zu, y);
      if (keeps) {
        w.store_one(g, pitch_z, bi, bj, zg, through);
        w.store_one(u, pitch_z, bi, bj, zu, through);
      }
      w.store_one(c, pitch_c, bi, bj, y, through);
    });
  }
};

// Bound by what it moves, two values read and two or three stored for each of D's, and by the vector unit: some thirty operations, an exponential and a
// reciprocal a value, 18 us of a round of 256x256 tiles.  What is read is requested as far ahead as 32 registers hold (64 spill, and a tile in its spilled form
// took 67 us where it takes 40).  8192 x 2048 x 768 bf16, H again too: 49 us alone (3.9 TB/s), 61 to 65 among the gradient's other products, whose
// results have displaced what it reads (106 MB read, 101 written).
struct GatedGrad {
  typedef GatedArgs Args;
  static constexpr int MOVES = PLACE_ALL;
  static constexpr bool OWN_END = true, STAYS = false, DUAL = false;
  template <typename C>
  static __device__ __attribute__((always_inline)) void touch(const Args&, const TilePlace&, uint32_t (&)[2]) {}

  // (dG and dU may lie where G and U do: a lane reads what it will write, and before)
  template <typename C, typename Acc, typename Hook>
  static __device__ __attribute__((always_inline)) void finish(const Args& a, Acc (&acc)[C::MBLK][C::NBLK], const TilePlace& p, Hook&&) {
    constexpr int MB = C::MB, NACC = MB * MB / 64;
    typedef WaveBlocks<C, C::NBLK> W;
    const int rows = min(C::BM, a.M - p.m0), cols = min(C::BN, a.N - p.n0);
    const W w{p.row, p.col, cols, p.lane};
    const uint32_t pitch_h = (uint32_t)(a.ldc * W::OS), pitch_z = (uint32_t)(a.ld_preact * W::OS), pitch_d = (uint32_t)(a.ld_dpreact * W::OS);
    const __amdgpu_buffer_rsrc_t h = tile_matrix(a.C, a.ldc, p.m0, p.n0, rows, cols, W::OS);
    const __amdgpu_buffer_rsrc_t g = tile_matrix(a.preact, a.ld_preact, p.m0, p.n0, rows, cols, W::OS);
    const __amdgpu_buffer_rsrc_t u = tile_matrix((char*)a.preact + a.far_preact * W::OS, a.ld_preact, p.m0, p.n0, rows, cols, W::OS);
    const __amdgpu_buffer_rsrc_t dg = tile_matrix(a.dpreact, a.ld_dpreact, p.m0, p.n0, rows, cols, W::OS);
    const __amdgpu_buffer_rsrc_t du = tile_matrix((char*)a.dpreact + a.far_dpreact * W::OS, a.ld_dpreact, p.m0, p.n0, rows, cols, W::OS);
    const bool again = a.C != nullptr, through = a.through;
    const ActForm form(a.act);
    // x: G, then dG; y: U, then dU; z: C.  The value and the slope of gelu and silu come from one exponential.
    auto compute = [&](auto bi, auto bj, auto first, auto& x, auto& y, auto& z) GENSOR_INLINE {
      constexpr int N = sizeof(x) / sizeof(float);
      auto each = [&](auto&& value_and_slope) GENSOR_INLINE {
#pragma unroll
        for (int v = 0; v < N; ++v) {
          const float d = a.alpha * acc[bi][bj][first + v], u = y[v];
          float value, slope;
          value_and_slope(x[v], value, slope);
          z[v] = value * u;
          x[v] = d * u * slope;
          y[v] = d * value;
        }
      };
      if (a.act == ACT_NONE) {
        each([&](float g, float& value, float& slope) GENSOR_INLINE { value = g; slope = 1.f; });
      } else if (a.act == ACT_RELU) {
        each([&](float g, float& value, float& slope) GENSOR_INLINE { value = g < 0.f ? 0.f : g; slope = g > 0.f ? 1.f : 0.f; });
      } else {
        each([&](float g, float& value, float& slope) GENSOR_INLINE {
          float q;
          const float s = form.sigmoid(g, q);
          value = g * s;
          slope = fmaf(value * (1.f - s), fmaf(3.f * form.c2, q, form.c1), s);
        });
      }
    };
    // (every index is a constant: accumulators that are indexed in a loop would lie in memory)
    if (W::OS == 2 && a.paired) {
      constexpr int UNITS = C::MBLK * (C::NBLK / W::GB), EACH = W::HALVES * W::RS;
      constexpr int AHEAD = UNITS * EACH <= 16 ? UNITS : EACH >= 16 ? 1 : 16 / EACH;
      uint32_t in_g[AHEAD][W::HALVES][W::RS], in_u[AHEAD][W::HALVES][W::RS];
      static_for<AHEAD>([&](auto n) GENSOR_INLINE {
        w.request_pair(g, pitch_z, n % C::MBLK, n / C::MBLK * W::GB, in_g[n]);
        w.request_pair(u, pitch_z, n % C::MBLK, n / C::MBLK * W::GB, in_u[n]);
      });
      static_for<UNITS>([&](auto n) GENSOR_INLINE {
        constexpr std::integral_constant<int, n % C::MBLK> bi{};
        constexpr int bj = n / C::MBLK * W::GB, next = n + AHEAD;
        uint32_t got_g[W::HALVES][W::RS], got_u[W::HALVES][W::RS];
        static_for<W::HALVES * W::RS>([&](auto i) GENSOR_INLINE {
          got_g[i / W::RS][i % W::RS] = in_g[n % AHEAD][i / W::RS][i % W::RS];
          got_u[i / W::RS][i % W::RS] = in_u[n % AHEAD][i / W::RS][i % W::RS];
        });
        if constexpr (next < UNITS) {
          w.request_pair(g, pitch_z, next % C::MBLK, next / C::MBLK * W::GB, in_g[n % AHEAD]);
          w.request_pair(u, pitch_z, next % C::MBLK, next / C::MBLK * W::GB, in_u[n % AHEAD]);
        }
        const uint32_t at_g = w.at_pair(pitch_d, bi, bj), at_u = w.at_pair(pitch_d, bi, bj), at_h = w.at_pair(pitch_h, bi, bj);
        static_for<W::HALVES>([&](auto half) GENSOR_INLINE {
          float x[W::GB][2], y[W::GB][2], z[W::GB][2];
          w.received_half(got_g[half], x);
          w.received_half(got_u[half], y);
          static_for<W::GB>([&](auto i) GENSOR_INLINE { compute(bi, std::integral_constant<int, bj + i>{}, std::integral_constant<int, 2 * half>{}, x[i], y[i], z[i]); });
          w.store_half(dg, pitch_d, at_g, half, x, through);
          w.store_half(du, pitch_d, at_u, half, y, through);
          if (again) w.store_half(h, pitch_h, at_h, half, z, through);
        });
      });
      return;
    }
    constexpr int BLOCKS = C::MBLK * C::NBLK, AHEAD = BLOCKS * NACC <= 16 ? BLOCKS : 16 / NACC;
    uint32_t in_g[AHEAD][NACC], in_u[AHEAD][NACC];
    static_for<AHEAD>([&](auto n) GENSOR_INLINE {
      w.request_one(g, pitch_z, n % C::MBLK, n / C::MBLK, in_g[n]);
      w.request_one(u, pitch_z, n % C::MBLK, n / C::MBLK, in_u[n]);
    });
    static_for<BLOCKS>([&](auto n) GENSOR_INLINE {
      constexpr std::integral_constant<int, n % C::MBLK> bi{};
      constexpr std::integral_constant<int, n / C::MBLK> bj{};
      constexpr int next = n + AHEAD;
      float x[NACC], y[NACC], z[NACC];
      w.received_one(in_g[n % AHEAD], x);
      w.received_one(in_u[n % AHEAD], y);
      if constexpr (next < BLOCKS) {
        w.request_one(g, pitch_z, next % C::MBLK, next / C::MBLK, in_g[n % AHEAD]);
        w.request_one(u, pitch_z, next % C::MBLK, next / C::MBLK, in_u[n % AHEAD]);
      }
      compute(bi, bj, std::integral_constant<int, 0>{}, x, y, z);
      w.store_one(dg, pitch_d, bi, bj, x, through);
      w.store_one(du, pitch_d, bi, bj, y, through);
      if (again) w.store_one(h, pitch_h, bi, bj, z, through);
    });
  }
};

// x of every lane group of a block (rows 4 apart) joined: all of them hold the result
template <int MB, typename Op>
__device__ __attribute__((always_inline)) inline float over_groups(float x, Op&& op) {
  if constexpr (MB == 16) {
    const auto q = __builtin_amdgcn_permlane16_swap(as_u32(x), as_u32(x), false, false);
    const uint32_t q0 = q[0], q1 = q[1];
    x = op(as_f32(q0), as_f32(q1));
  }
  const auto q = __builtin_amdgcn_permlane32_swap(as_u32(x), as_u32(x), false, false);
  const uint32_t q0 = q[0], q1 = q[1];
  return op(as_f32(q0), as_f32(q1));
}

// The logits' reduction of END_LSE with one more sum, and, for the largest entries, the maxima of sets of 32 rows and the logits of the sets whose
// maximum is above the token's bar (46 of 768 in the second of three pieces, 6 of 675 in the third).  Sums and maxima of a token lie side by side for the wave that joins them.
// Bound by the products under the power limit (16 of a tile's 21 to 24 us), then by the vector unit.  4096 tokens over 50257 entries of width 768, f16, us
// with the join: lse 268 (1.18 PFLOP/s), with entropy 277, with the log probabilities of targets 278, with eight alternatives 311, all together 333 (three
// pieces; matrix units busy 45 %; 316 to 352 from card to card); one token 17.4, which is reading W at 4.4 TB/s.
struct Score {
  typedef ScoreArgs Args;
  static constexpr int MOVES = PLACE_ALL;
  static constexpr bool OWN_END = true, STAYS = true, DUAL = false;
  template <typename C>
  static __device__ __attribute__((always_inline)) void touch(const Args&, const TilePlace&, uint32_t (&)[2]) {}

  template <typename C, typename Acc, typename Hook>
  static __device__ __attribute__((always_inline)) void finish(const Args& a, Acc (&acc)[C::MBLK][C::NBLK], const TilePlace& p, Hook&& before_stores) {
    constexpr int MB = C::MB, NACC = MB * MB / 64;
    constexpr int SET = score_set(C::WM), SETS = C::WM / SET, PER = SET / MB;      // blocks of a set
    constexpr float log2e = 1.44269504088896340736f, ln2 = 0.69314718055994530942f;
    const int lane = p.lane, frow = lane % MB, fgrp = lane / MB;
    const int first = p.m0 + p.row;                                  // the wave's first row
    const int rows = min(C::WM, a.M - first);
    const int slab = first / C::WM;
    float tops[C::NBLK], sums[C::NBLK], rests[C::NBLK], at_target[C::NBLK], set_top[C::NBLK][SETS], bar[C::NBLK];
    bool hit[C::NBLK];
    // (asked for early: nothing waits for it until everything is computed)
#pragma unroll
    for (int bj = 0; bj < C::NBLK; ++bj) {
      const int token = p.n0 + p.col + bj * MB + frow;
      bar[bj] = a.bar && token < a.N ? a.bar[token] : NAN;
    }
    if (a.alpha != 1.f) {
#pragma unroll
      for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
        for (int bj = 0; bj < C::NBLK; ++bj)
#pragma unroll
          for (int v = 0; v < NACC; ++v) acc[bi][bj][v] *= a.alpha;
    }
    if (rows < C::WM) {
#pragma unroll
      for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
        for (int v = 0; v < NACC; ++v)
          if (bi * MB + block_row_of<C>(v) + 4 * fgrp >= rows)
#pragma unroll
            for (int bj = 0; bj < C::NBLK; ++bj) acc[bi][bj][v] = -INFINITY;
    }
    auto larger = [](float x, float y) { return fmaxf(x, y); };
    auto plus = [](float x, float y) { return x + y; };
#pragma unroll
    for (int bj = 0; bj < C::NBLK; ++bj) {
      const int token = p.n0 + p.col + bj * MB + frow;
      const bool there = token < a.N;
      float top = -INFINITY;
#pragma unroll
      for (int s = 0; s < SETS; ++s) {
        float t = -INFINITY;
#pragma unroll
        for (int b = 0; b < PER; ++b)
#pragma unroll
          for (int v = 0; v < NACC; ++v) t = fmaxf(t, acc[s * PER + b][bj][v]);
        set_top[bj][s] = over_groups<MB>(t, larger);
        top = fmaxf(top, set_top[bj][s]);
      }
      // exp(z - ref) = 2^y, y = log2(e) z - (log2(e) ref rounded), all terms off by one factor 2^off, which is taken out of the sums.  (off is up to 2^-24 of
      // that product.  Beyond 1e6 the difference is taken first: from there on the weights would be mostly off, and beyond 1e9 its power may be no number; a
      // stretch of the vocabulary that is shut off with large negative logits comes here, too.  The column's own choice, so that a token's bits do not depend
      // on its neighbours.)  The weight in the second sum is y itself; where a logit is minus infinity, or a row none, that is 0 times minus infinity,
      // and the sums are taken again with weights that are held above -1e4.
      const float ref = lse_reference(top);
      const bool far = fabsf(ref) > 1e6f;
      const float base = far ? 0.f : -(log2e * ref), off = far ? 0.f : fmaf(log2e, ref, base);
      float sum = 0.f, rest = 0.f;
      auto reduce = [&](auto weighted_tag, auto&& exponent, auto&& weight) {
        constexpr bool weighted = decltype(weighted_tag)::value;
        sum = rest = 0.f;
#pragma unroll
        for (int bi = 0; bi < C::MBLK; ++bi) {
          float part = 0.f, more = 0.f;
#pragma unroll
          for (int v = 0; v < NACC; ++v) {
            const float y = exponent(acc[bi][bj][v]), e = __builtin_amdgcn_exp2f(y);
            part += e;
            if constexpr (weighted) more = fmaf(e, weight(y), more);
          }
          sum += part;
          rest += more;
        }
      };
      auto near_ref = [&](float z) { return fmaf(log2e, z, base); };
      auto any_ref = [&](float z) { return far ? log2e * (z - ref) : fmaf(log2e, z, base); };
      auto itself = [](float y) { return y; };
      auto finite = [](float y) { return fmaxf(y, -1e4f); };
      if (!a.weighted) {
        if (__any(far)) reduce(std::false_type{}, any_ref, itself);
        else reduce(std::false_type{}, near_ref, itself);
      } else {
        if (__any(far)) reduce(std::true_type{}, any_ref, finite);
        else reduce(std::true_type{}, near_ref, itself);
        if (__any(rest != rest)) reduce(std::true_type{}, any_ref, finite);
      }
      rest = ln2 * fmaf(-off, sum, rest) * __builtin_amdgcn_exp2f(-off);
      sum *= __builtin_amdgcn_exp2f(-off);
      tops[bj] = top;
      sums[bj] = over_groups<MB>(sum, plus);
      rests[bj] = over_groups<MB>(rest, plus);
      hit[bj] = false;
      at_target[bj] = 0.f;
      if (a.targets) {
        const int64_t target = there ? a.targets[token] : -1;
        const int64_t entry = (int64_t)first + a.row_first;
        const int at = there && target != a.ignore && target >= entry && target < entry + rows ? (int)(target - entry) - 4 * fgrp : -1;
        if (__any(at >= 0)) {
#pragma unroll
          for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
            for (int v = 0; v < NACC; ++v)
              if (at == bi * MB + block_row_of<C>(v)) {
                hit[bj] = true;
                at_target[bj] = acc[bi][bj][v];
              }
        }
      }
    }
    before_stores();
    if (rows <= 0) return;
#pragma unroll
    for (int bj = 0; bj < C::NBLK; ++bj) {
      const int token = p.n0 + p.col + bj * MB + frow;
      if (token < a.N && fgrp == 0) {
        a.parts[(int64_t)token * a.slabs + slab] = f32x4{tops[bj], sums[bj], rests[bj], 0.f};
        if (a.sets) {
          typedef float maxima_t __attribute__((ext_vector_type(SETS)));
          maxima_t m;
#pragma unroll
          for (int s = 0; s < SETS; ++s) m[s] = set_top[bj][s];
          *(maxima_t*)(a.set_max + (int64_t)token * a.sets + slab * SETS) = m;
        }
      }
      if (hit[bj]) a.at_target[token] = at_target[bj];
    }
    if (!a.sets) return;
#pragma unroll
    for (int bj = 0; bj < C::NBLK; ++bj) {
      const int token = p.n0 + p.col + bj * MB + frow;
      const bool there = token < a.N;
      if (!__any(there && set_is_stored(tops[bj], bar[bj]))) continue;
#pragma unroll
      for (int s = 0; s < SETS; ++s)
        if (there && set_is_stored(set_top[bj][s], bar[bj])) {
          float* to = a.logits + ((int64_t)token * a.sets + slab * SETS + s) * SET + 4 * fgrp;
#pragma unroll
          for (int b = 0; b < PER; ++b)
#pragma unroll
            for (int q = 0; q < NACC / 4; ++q) {
              const auto& x = acc[s * PER + b][bj];
              *(f32x4*)(to + b * MB + 8 * q) = f32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
            }
        }
    }
  }
};

// Weights of zero are a choice, not a factor: the logits of a token that teaches nothing may be infinite or NaN.  G is rounded to the type because it is an
// operand of two products, which run at nine times fp32's rate so (bf16: dX and dW 0.0023 from 64 bits, 0.0017 with fp32 throughout).  Bound as END_PROB is: 4096 tokens over
// 50257 entries of width 768, bf16, 186 and 122 us of two pieces (1.03 PFLOP/s, matrix units busy 45 %, 412 MB written).
struct Teach {
  typedef FusedArgs Args;
  static constexpr int MOVES = PLACE_ALL;
  static constexpr bool OWN_END = true, STAYS = false, DUAL = false;
  template <typename C>
  static __device__ __attribute__((always_inline)) void touch(const Args&, const TilePlace&, uint32_t (&)[2]) {}

  template <typename C, typename Acc, typename Hook>
  static __device__ __attribute__((always_inline)) void finish(const Args& a, Acc (&acc)[C::MBLK][C::NBLK], const TilePlace& p, Hook&&) {
    constexpr int MB = C::MB, NACC = MB * MB / 64;
    typedef Fused<END_LINEAR, MOVE_NONE> Plain;
    const float scale = a.scale ? *a.scale : 1.f;
    if (a.alpha != 1.f) {
#pragma unroll
      for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
        for (int bj = 0; bj < C::NBLK; ++bj)
#pragma unroll
          for (int v = 0; v < NACC; ++v) acc[bi][bj][v] *= a.alpha;
    }
#pragma unroll
    for (int bj = 0; bj < C::NBLK; ++bj) {
      const int token = p.n0 + p.col + bj * MB + p.lane % MB;
      const bool there = token < a.tokens;
      const float weight = there ? a.dloss[token] * scale : 0.f;
      const bool counts = weight != 0.f;
      const float lse = counts ? a.lse[token] : INFINITY, base = Plain::template below_lse<C>(acc, bj, lse, counts);
#pragma unroll
      for (int bi = 0; bi < C::MBLK; ++bi)
#pragma unroll
        for (int v = 0; v < NACC; ++v) acc[bi][bj][v] = counts ? weight * Plain::template probability<C>(acc[bi][bj][v], lse, base) : 0.f;
    }
    Plain::template finish_linear<C, false>(a, acc, p);
  }
};

}  // namespace gensor
