// Tile kernels of kind kWeight (tile_gemm.cuh).
#include "tile_gemm.cuh"

namespace bkmoo {

const void* tile_weight_fn(int cg) {
  return cg == 1 ? (const void*)tile_gemm_kernel<kWeight, 1> : (const void*)tile_gemm_kernel<kWeight, 2>;
}

}  // namespace bkmoo
