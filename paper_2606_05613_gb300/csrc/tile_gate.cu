// Tile kernels of kind kGate (tile_gemm.cuh).
#include "tile_gemm.cuh"

namespace bkmoo {

const void* tile_gate_fn(int cg, int bn) {
  if (cg == 2) return (const void*)tile_gemm_kernel<kGate, 2, 256, kPlain>;
  if (bn == 256) return (const void*)tile_gemm_kernel<kGate, 1, 256, kPlain>;
  if (bn == 128) return (const void*)tile_gemm_kernel<kGate, 1, 128, kPlain>;
  return (const void*)tile_gemm_kernel<kGate, 1, 64, kPlain>;
}

}  // namespace bkmoo
