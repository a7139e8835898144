// Tables of the compiled ends of lm_kernel.hpp: what the tiles of fused_registry.hpp also exist with, and the tiles of two products at once.
#pragma once
#include "fused_registry.hpp"
#include "lm_kernel.hpp"

namespace gensor {

typedef hipError_t (*ScoreLaunch)(const ScoreArgs&, hipStream_t);
typedef hipError_t (*GatedLaunch)(const GatedArgs&, hipStream_t);

// beside g_fused, tile by tile (null: not compiled)
struct LmEnds {
  ScoreLaunch score;
  FusedLaunch teach;
  GatedLaunch gated_grad;
};
extern const LmEnds g_lm_ends[];

// (a tile's bn columns are bn / 2 of either product)
struct GatedDesc {
  InstanceDesc d;
  GatedLaunch launch;
};
extern const GatedDesc g_gated[];
extern const int g_num_gated;

template <typename C, typename F>
hipError_t launch_end(const typename F::Args& a, hipStream_t st) {
  static std::atomic<uint64_t> done{0};
  hipError_t e = allow_dynamic_lds(contraction_kernel<C, false, false, false, F>, C::LDS_BYTES, done);
  if (e != hipSuccess) return e;
  const unsigned tiles = (unsigned)a.tiles_m * (unsigned)a.tiles_n;
  // (workgroups of the alternating tiles stay for further tiles: one to a compute unit)
  const unsigned most = C::ALTERNATE && F::STAYS ? 256u : 0xffffffffu;
  hipLaunchKernelGGL((contraction_kernel<C, false, false, false, F>), dim3(tiles < most ? tiles : most), dim3(C::THREADS), C::LDS_BYTES, st, a);
  return hipGetLastError();
}

}  // namespace gensor
