// Tile kernels of kind kWeight, fp32 results (tile_gemm.cuh).
#include "tile_gemm.cuh"

namespace bkmoo {
namespace {

template <int MODE>
const void* fn(int bn) {
  return bn == 128 ? (const void*)tile_gemm_kernel<kWeight, 1, 128, MODE>
                   : (const void*)tile_gemm_kernel<kWeight, 1, 64, MODE>;
}

}  // namespace

const void* tile_weight_f32_fn(int bn, int mode) {
  return mode == kSums         ? fn<kSums>(bn)
         : mode == kSumsAdded  ? fn<kSumsAdded>(bn)
         : mode == kSumsTurned ? fn<kSumsTurned>(bn)
                               : fn<kSumsTurnedAdded>(bn);
}

}  // namespace bkmoo
