// Tile kernels of kind kBoth, plain (tile_gemm.cuh); the other modes in
// tile_both_bf16.cu and tile_both_f32.cu (nvcc runs them side by side).
#include "tile_gemm.cuh"

namespace bkmoo {

const void* tile_both_bf16_fn(int cg, int bn, bool turned);
const void* tile_both_f32_fn(int bn, int mode);

const void* tile_both_fn(int cg, int bn, int mode) {
  if (mode_f32(mode)) return tile_both_f32_fn(bn, mode);
  if (mode != kPlain) return tile_both_bf16_fn(cg, bn, mode_turned(mode));
  if (cg == 2) return (const void*)tile_gemm_kernel<kBoth, 2, 256, kPlain>;
  if (bn == 256) return (const void*)tile_gemm_kernel<kBoth, 1, 256, kPlain>;
  if (bn == 128) return (const void*)tile_gemm_kernel<kBoth, 1, 128, kPlain>;
  return (const void*)tile_gemm_kernel<kBoth, 1, 64, kPlain>;
}

}  // namespace bkmoo
