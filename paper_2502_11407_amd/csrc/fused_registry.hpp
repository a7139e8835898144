// Table of the compiled tiles of the products that are consumed in place (fused_kernel.hpp): for each tile the launches of
// the ends and groupings it exists with.
#pragma once
#include "fused_kernel.hpp"
#include "registry.hpp"

namespace gensor {

enum { FUSED_LINEAR = 0, FUSED_LINEAR_SPLIT = 1, FUSED_ROWS = 2, FUSED_DEPTH = 3, FUSED_LSE = 4, FUSED_PROB = 5, FUSED_KINDS = 6 };

typedef hipError_t (*FusedLaunch)(const FusedArgs&, hipStream_t);

struct FusedDesc {
  InstanceDesc d;
  FusedLaunch launch[FUSED_KINDS];         // null: not compiled
};

extern const FusedDesc g_fused[];
extern const int g_num_fused;

// (grouped rows: tiles_m counts the tile rows that there can be at most, over all groups)
template <typename C, int END, int MOVE, bool SPLIT = false>
hipError_t launch_fused(const FusedArgs& a, hipStream_t st) {
  if constexpr (C::HAS_NARROW && END == END_LINEAR && MOVE == MOVE_NONE && !SPLIT) {
    if (a.narrow) return launch_fused<NarrowCfg<C>, END, MOVE>(a, st);
  }
  typedef Fused<END, MOVE> F;
  static std::atomic<uint64_t> done{0};
  hipError_t e = allow_dynamic_lds(contraction_kernel<C, SPLIT, false, false, F>, C::LDS_BYTES, done);
  if (e != hipSuccess) return e;
  const unsigned tiles = (unsigned)a.tiles_m * (unsigned)a.tiles_n * (unsigned)a.batch;
  // (workgroups of the alternating tiles stay for further tiles: one to a compute unit)
  const unsigned most = C::ALTERNATE && F::STAYS ? 256u : 0xffffffffu;
  const unsigned grid = SPLIT ? (unsigned)a.whole + (tiles - (unsigned)a.whole) * (unsigned)a.split : tiles < most ? tiles : most;
  hipLaunchKernelGGL((contraction_kernel<C, SPLIT, false, false, F>), dim3(grid), dim3(C::THREADS), C::LDS_BYTES, st, a);
  return hipGetLastError();
}

}  // namespace gensor
