// Tile kernels of kind kWeight (tile_gemm.cuh).
#include "tile_gemm.cuh"

namespace bkmoo {
namespace {

template <bool TURN>
const void* fn(int cg, int bn) {
  if (cg == 2) return (const void*)tile_gemm_kernel<kWeight, 2, 256, TURN>;
  if (bn == 256) return (const void*)tile_gemm_kernel<kWeight, 1, 256, TURN>;
  if (bn == 128) return (const void*)tile_gemm_kernel<kWeight, 1, 128, TURN>;
  return (const void*)tile_gemm_kernel<kWeight, 1, 64, TURN>;
}

}  // namespace

const void* tile_weight_fn(int cg, int bn, bool turn) { return turn ? fn<true>(cg, bn) : fn<false>(cg, bn); }

}  // namespace bkmoo
