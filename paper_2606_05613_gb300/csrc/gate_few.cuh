// The gated projections for a few rows (gate_few.cu).
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace bkmoo {

constexpr int kFewRows = 8;

struct FewArgs {
  const __nv_bfloat16 *x, *wg, *wu;
  __nv_bfloat16 *h, *a, *b;     // h, or a and b, may be NULL
  int64_t ldx, ldw, ldh, ld_ab;
  int32_t T, D, F, act;
};
cudaError_t launch_gate_few(const FewArgs& p, int sms, cudaStream_t s);

}  // namespace bkmoo
