// Tile kernels of kind kBoth, bf16 results added to what is there or not in whole
// aligned pieces (tile_gemm.cuh).
#include "tile_gemm.cuh"

namespace bkmoo {
namespace {

template <int MODE>
const void* fn(int cg, int bn) {
  if (cg == 2) return (const void*)tile_gemm_kernel<kBoth, 2, 256, MODE>;
  if (bn == 256) return (const void*)tile_gemm_kernel<kBoth, 1, 256, MODE>;
  if (bn == 128) return (const void*)tile_gemm_kernel<kBoth, 1, 128, MODE>;
  return (const void*)tile_gemm_kernel<kBoth, 1, 64, MODE>;
}

}  // namespace

const void* tile_both_bf16_fn(int cg, int bn, bool turned) {
  return turned ? fn<kTurned>(cg, bn) : fn<kAdded>(cg, bn);
}

}  // namespace bkmoo
