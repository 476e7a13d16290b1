// Tile kernels of kind kBoth, bf16 results added to what is there or not in whole
// aligned pieces (tile_gemm.cuh).
#include "tile_gemm.cuh"

namespace bkmoo {
namespace {

// (of 128 columns at most where results are turned: tile_shape)
const void* added_fn(int cg, int bn) {
  if (cg == 2) return (const void*)tile_gemm_kernel<kBoth, 2, 256, kAdded>;
  if (bn == 256) return (const void*)tile_gemm_kernel<kBoth, 1, 256, kAdded>;
  if (bn == 128) return (const void*)tile_gemm_kernel<kBoth, 1, 128, kAdded>;
  return (const void*)tile_gemm_kernel<kBoth, 1, 64, kAdded>;
}
const void* turned_fn(int bn) {
  return bn == 128 ? (const void*)tile_gemm_kernel<kBoth, 1, 128, kTurned>
                   : (const void*)tile_gemm_kernel<kBoth, 1, 64, kTurned>;
}

}  // namespace

const void* tile_both_bf16_fn(int cg, int bn, bool turned) {
  return turned ? turned_fn(bn) : added_fn(cg, bn);
}

}  // namespace bkmoo
