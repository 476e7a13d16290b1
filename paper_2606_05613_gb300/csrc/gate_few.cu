// The gated projections for a few rows of x (serving): h = act(x Wg^T) (x Wu^T).
//
// Bound by the weights' bytes, each of which is used for at most 32 rows: they go
// from memory straight into registers, 16 bytes a lane, with no stop in shared
// memory, and warp-wide products (mma m16n8k16, fp32 sums) do the arithmetic: 16
// weight rows, 8 of Wg over the same 8 of Wu, by 8 rows of x, so that a lane ends
// with a and b of the same place.  A product's 16 steps of the sum may be any 16 as
// long as both operands agree: a lane takes 8 consecutive elements of its weight
// row and of its x row, its part of two products' steps.
//
// A CTA does 8 columns of h.  Its 1 to 8 warps share the sum over the width, a
// window of 64 each in turn, and join in shared memory in a fixed order: as many
// as let all CTAs of the grid be resident at once, so that the weights stream in
// without a pause for CTAs that come and go (CTAs of 8 warps in several waves:
// 2048 -> 8192 17.1 us, 4096 -> 12288 43.4).  The x row comes with each window,
// as far ahead as the weights: fetched when it is used, its way from L2 is what a
// warp waits for (22.8 and 68 us).
#include "gate_few.cuh"

#include "tile_gemm.cuh"

namespace bkmoo {
namespace {

constexpr int kFewWindow = 64;      // of the sum: 128 bytes of a row, 32 a lane
constexpr int kFewAhead = 2;        // windows of a warp in flight
// Warps of an SM.  2 windows ahead of 24 warps: 2048 -> 8192 13.7 us, 4096 -> 12288
// 33.7 (4.9 and 5.97 TB/s); 4 of 16 13.1, 37.5; 2 of 32, which spills, 14.2, 36.6;
// windows of 32, 64 bytes of a row at a time, 4 of 24 14.7, 34.7.
// (x takes the registers of 8 of them from 9 rows on.)
constexpr int few_resident(int nt) { return nt == 1 ? 24 : 16; }

// Elements k to k + 7 of a row of D, zeros beyond its end.  (Not by the read-only path:
// the kernel may begin before the one that writes x or the weights has ended.)
template <bool STREAM>
__device__ __forceinline__ uint4 load8(const __nv_bfloat16* row, int k, int D) {
  if (k + 8 <= D) {
    const uint4* p = reinterpret_cast<const uint4*>(row + k);
    uint4 v;
    if (STREAM)
      asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                   : "l"(p)
                   : "memory");
    else
      asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                   : "l"(p)
                   : "memory");
    return v;
  }
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (k + j < D) w[j / 2] |= (uint32_t)__bfloat16_as_ushort(row[k + j]) << (16 * (j & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void product16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                          uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// WARPS share the sum; NT groups of 8 rows of x.
template <int WARPS, int NT>
__global__ void __launch_bounds__(32 * WARPS, few_resident(NT) / WARPS) gate_few_kernel(const FewArgs p) {
  grid_wait();
  const int wid = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int f0 = blockIdx.x * 8;
  const bool wlive = f0 + g < p.F;
  const __nv_bfloat16 *wg = p.wg + (int64_t)(wlive ? f0 + g : 0) * p.ldw,
                      *wu = p.wu + (int64_t)(wlive ? f0 + g : 0) * p.ldw;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  const int windows = (p.D + kFewWindow - 1) / kFewWindow;
  uint4 ag[kFewAhead][2], au[kFewAhead][2], b[kFewAhead][2][NT];
  auto fetch = [&](int i, int w) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = kFewWindow * w + 16 * q + 8 * h;
      ag[i][h] = wlive && w < windows ? load8<true>(wg, k, p.D) : zero;
      au[i][h] = wlive && w < windows ? load8<true>(wu, k, p.D) : zero;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int t = 8 * n + g;
        b[i][h][n] = t < p.T && w < windows ? load8<false>(p.x + t * p.ldx, k, p.D) : zero;
      }
    }
  };
#pragma unroll
  for (int i = 0; i < kFewAhead; ++i) fetch(i, wid + i * WARPS);
  float c[NT][4] = {};
  for (int w0 = wid; w0 < windows; w0 += WARPS * kFewAhead) {
#pragma unroll
    for (int i = 0; i < kFewAhead; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          product16(c[n], ag[i][h].x, au[i][h].x, ag[i][h].y, au[i][h].y, b[i][h][n].x, b[i][h][n].y);
          product16(c[n], ag[i][h].z, au[i][h].z, ag[i][h].w, au[i][h].w, b[i][h][n].z, b[i][h][n].w);
        }
      }
      fetch(i, w0 + (i + kFewAhead) * WARPS);
    }
  }
  __shared__ float part[WARPS][2][8 * NT][8];     // [a or b][row of x][column]
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    part[wid][0][8 * n + 2 * q][g] = c[n][0];
    part[wid][0][8 * n + 2 * q + 1][g] = c[n][1];
    part[wid][1][8 * n + 2 * q][g] = c[n][2];
    part[wid][1][8 * n + 2 * q + 1][g] = c[n][3];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * NT; i += 32 * WARPS) {
    const int t = i >> 3, f = i & 7, col = f0 + f;
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      a += part[w][0][t][f];
      b += part[w][1][t][f];
    }
    if (t >= p.T || col >= p.F) continue;
    if (p.h) p.h[t * p.ldh + col] = __float2bfloat16_rn(activation(p.act, a) * b);
    if (p.a) {
      p.a[t * p.ld_ab + col] = __float2bfloat16_rn(a);
      p.b[t * p.ld_ab + col] = __float2bfloat16_rn(b);
    }
  }
}

template <int NT>
const void* few_fn(int warps) {
  return warps == 1   ? (const void*)gate_few_kernel<1, NT>
         : warps == 2 ? (const void*)gate_few_kernel<2, NT>
         : warps == 4 ? (const void*)gate_few_kernel<4, NT>
                      : (const void*)gate_few_kernel<8, NT>;
}

}  // namespace

cudaError_t launch_gate_few(const FewArgs& p, int sms, cudaStream_t s) {
  const int units = (p.F + 7) / 8, windows = (p.D + kFewWindow - 1) / kFewWindow;
  const int nt = p.T <= 8 ? 1 : p.T <= 16 ? 2 : 4;
  const int64_t most = (int64_t)sms * few_resident(nt);
  // (a warp keeps two windows at least)
  int warps = 1;
  while (warps < 8 && (int64_t)units * warps * 2 <= most && windows >= 4 * warps) warps *= 2;
  FewArgs q = p;
  void* list[] = {&q};
  return launch_behind(nt == 1 ? few_fn<1>(warps) : nt == 2 ? few_fn<2>(warps) : few_fn<4>(warps),
                       dim3(units), dim3(32 * warps), list, 0, s, true);
}

}  // namespace bkmoo
