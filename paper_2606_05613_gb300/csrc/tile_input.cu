// Tile kernels of kind kInput (tile_gemm.cuh).
#include "tile_gemm.cuh"

namespace bkmoo {

const void* tile_input_fn(int cg) {
  return cg == 1 ? (const void*)tile_gemm_kernel<kInput, 1> : (const void*)tile_gemm_kernel<kInput, 2>;
}

}  // namespace bkmoo
