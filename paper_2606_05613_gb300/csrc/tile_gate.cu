// Tile kernels of kind kGate (tile_gemm.cuh).
#include "tile_gemm.cuh"

namespace bkmoo {

const void* tile_gate_fn(int cg) {
  return cg == 1 ? (const void*)tile_gemm_kernel<kGate, 1> : (const void*)tile_gemm_kernel<kGate, 2>;
}

}  // namespace bkmoo
