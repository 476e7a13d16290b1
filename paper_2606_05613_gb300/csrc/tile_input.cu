// Tile kernels of kind kInput (tile_gemm.cuh).
#include "tile_gemm.cuh"

namespace bkmoo {

const void* tile_input_fn(int cg, int bn) {
  if (cg == 2) return (const void*)tile_gemm_kernel<kInput, 2, 256>;
  if (bn == 256) return (const void*)tile_gemm_kernel<kInput, 1, 256>;
  if (bn == 128) return (const void*)tile_gemm_kernel<kInput, 1, 128>;
  return (const void*)tile_gemm_kernel<kInput, 1, 64>;
}

}  // namespace bkmoo
