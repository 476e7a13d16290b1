// The gated projections for a few rows (gate_few.cu).
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace bkmoo {

// Whether T rows are few (against the tile kernel, steady, us: 16 rows 1024 -> 2816 4.4
// / 7.4, 2909 -> 2782 11.2 / 12.1, 2048 -> 8192 14.3 / 14.5, 4096 -> 12288 44 / 37; 32
// rows 1024 -> 2816 5.9 / 7.4, 384 -> 9728 6.7 / 8.6, 2909 -> 2782 15.2 / 12.1, 2048 ->
// 8192 18.3 / 14.5): every 8 columns read x again, so the more rows, the less weights.
inline bool few_rows(int64_t T, int64_t D, int64_t F) {
  const double weights = 4.0 * (double)D * (double)F;      // bytes
  return T <= 8 || (T <= 16 && weights <= 70e6) || (T <= 32 && weights <= 20e6);
}

struct FewArgs {
  const __nv_bfloat16 *x, *wg, *wu;
  __nv_bfloat16 *h, *a, *b;     // h, or a and b, may be NULL
  int64_t ldx, ldw, ldh, ld_ab;
  int32_t T, D, F, act;
};
cudaError_t launch_gate_few(const FewArgs& p, int sms, cudaStream_t s);

}  // namespace bkmoo
