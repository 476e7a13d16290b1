// Tile kernels of kind kBoth (tile_gemm.cuh).
#include "tile_gemm.cuh"

namespace bkmoo {

const void* tile_both_fn(int cg, int bn) {
  if (cg == 2) return (const void*)tile_gemm_kernel<kBoth, 2, 256>;
  if (bn == 256) return (const void*)tile_gemm_kernel<kBoth, 1, 256>;
  if (bn == 128) return (const void*)tile_gemm_kernel<kBoth, 1, 128>;
  return (const void*)tile_gemm_kernel<kBoth, 1, 64>;
}

}  // namespace bkmoo
