// One AdamW step over all the tensors of a model (include/bkmoo.h), and the norm
// it clips by.
//
// The direction, the moments and the master copy are flat, in the layout of the
// resolve; the weights are tensors of their own.  A warp takes 256 consecutive
// flat elements at a time, whatever tensors they lie in: each lane 4 and 4 more
// 128 further on, so that every access of the flat buffers is a whole vector and
// a warp's accesses are contiguous.  256 is also the block of elements that share
// a scale in 8 bits, so its largest value is a matter of one warp.  Which tensor
// an element belongs to comes from a table in the kernel's parameters (a binary
// search per four blocks, then steps).
//
// Bound by memory: per element the direction, the weight and both moments (and
// the master copy) are read once and written once.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cmath>

#include "common.cuh"

namespace bkmoo {
namespace {

constexpr int kBlock = 256;          // elements per scale, and per warp and turn
constexpr int kAdamTable = 1024;     // tensors a launch knows
constexpr int kAdamThreads = 256;
constexpr int kAdamTurns = 4;        // consecutive blocks of a warp
constexpr int64_t kAdamSpan = (int64_t)(kAdamThreads / 32) * kAdamTurns;   // blocks of a CTA

struct AdamArgs {
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;
  float* master;
  const float* norm;                 // NULL: neither clipped nor checked
  float max_norm;                    // 0: not clipped
  float b1, one_b1, b2, one_b2;
  float rate;                        // lr / (1 - beta1^step)
  float root;                        // 1 / sqrt(1 - beta2^step)
  float eps;
  uint64_t key;                      // of the rounding to 8 bits
  int64_t n;                         // flat elements
  int64_t first, blocks;             // this launch: blocks first .. first + blocks - 1
  int32_t tensors;
  void* p[kAdamTable];
  int64_t start[kAdamTable + 1];     // flat bounds of the tensors
  float keep[kAdamTable];            // 1 - lr weight_decay
};

__host__ __device__ inline uint64_t mix_word(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}
constexpr uint64_t kGold = 0x9E3779B97F4A7C15ull;

// Four consecutive elements, of which the first n exist (16-byte aligned base,
// index a multiple of 4).
__device__ __forceinline__ void load4(const float* p, int64_t i, int n, float (&x)[4]) {
  if (n >= 4) {
    const float4 t = __ldcs(reinterpret_cast<const float4*>(p + i));
    x[0] = t.x, x[1] = t.y, x[2] = t.z, x[3] = t.w;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = j < n ? p[i + j] : 0.0f;
  }
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, int64_t i, int n, float (&x)[4]) {
  if (n >= 4) {
    const uint2 t = __ldcs(reinterpret_cast<const uint2*>(p + i));
    x[0] = __uint_as_float(t.x << 16), x[1] = __uint_as_float(t.x & 0xffff0000u);
    x[2] = __uint_as_float(t.y << 16), x[3] = __uint_as_float(t.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = j < n ? __bfloat162float(p[i + j]) : 0.0f;
  }
}
__device__ __forceinline__ void store4(float* p, int64_t i, int n, const float (&x)[4]) {
  if (n >= 4) {
    __stcs(reinterpret_cast<float4*>(p + i), make_float4(x[0], x[1], x[2], x[3]));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[i + j] = x[j];
  }
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, int64_t i, int n, const float (&x)[4]) {
  if (n >= 4) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    __stcs(reinterpret_cast<uint2*>(p + i),
           make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b)));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[i + j] = __float2bfloat16_rn(x[j]);
  }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t i, int n) {
  if (n >= 4) return __ldcs(reinterpret_cast<const uint32_t*>(p + i));
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < n) w |= (uint32_t)p[i + j] << (8 * j);
  return w;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t i, int n, uint32_t w) {
  if (n >= 4) {
    __stcs(reinterpret_cast<uint32_t*>(p + i), w);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[i + j] = (uint8_t)(w >> (8 * j));
  }
}
__device__ __forceinline__ void decode4(uint32_t w, float scale, float (&x)[4]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> (16 * j)), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    x[2 * j] = f.x * scale;
    x[2 * j + 1] = f.y * scale;
  }
}

// |x| / scale as an e4m3 code, rounded up with the chance that the rest gives:
// u, 16 bits, stands for u / 65536.  2^-120 takes e4m3's smallest normal number,
// 2^-6, to fp32's, 2^-126, so the product's bits above the 20th are the code, of
// subnormal values too, and what is below them is the rest.
__device__ __forceinline__ uint32_t encode(float x, float inv, uint32_t u, bool positive) {
  const uint32_t bits = __float_as_uint(__fmul_rn(__fmul_rn(fabsf(x), inv), 0x1p-120f));
  uint32_t c = min((bits + (u << 4)) >> 20, 0x7eu);
  if (positive && c == 0 && bits > 0) c = 1;
  if (bits > 0x7f800000u) c = 0x7f;    // NaN stays NaN
  return c;
}

// The weights of four consecutive flat elements.
template <class P>
struct Weights {
  P* p;        // of the first element
  int t;       // its tensor
  int n;       // how many of the four lie in it
  float keep;
};
template <class P>
__device__ __forceinline__ Weights<P> find(const AdamArgs& a, int t, int64_t e) {
  while (t + 1 < a.tensors && a.start[t + 1] <= e) ++t;
  Weights<P> w;
  const int64_t s = a.start[t], left = a.start[t + 1] - e;
  w.p = static_cast<P*>(a.p[t]) + (e - s);
  w.t = t;
  w.n = left < 4 ? (int)left : 4;
  w.keep = a.keep[t];
  return w;
}

template <class P, class G, bool E4M3, bool MASTER>
__global__ void __launch_bounds__(kAdamThreads)
    adamw_kernel(const __grid_constant__ AdamArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t b0 = a.first + blockIdx.x * kAdamSpan + (threadIdx.x >> 5) * kAdamTurns;
  const int64_t end = a.first + a.blocks;
  if (b0 >= end) return;
  float clip = 1.0f;
  if (a.norm) {
    const float norm = *a.norm;
    if (!(fabsf(norm) <= 3.4028235e38f)) return;      // not a step to take
    if (a.max_norm > 0.0f) clip = fminf(1.0f, __fdiv_rn(a.max_norm, __fadd_rn(norm, 1e-6f)));
  }
  int t = 0;                        // the tensor of the first element
  {
    int hi = a.tensors;
    while (hi - t > 1) {
      const int mid = (t + hi) >> 1;
      if (a.start[mid] <= b0 * kBlock) t = mid;
      else hi = mid;
    }
  }
#pragma unroll 1
  for (int turn = 0; turn < kAdamTurns; ++turn) {
    const int64_t blk = b0 + turn;
    if (blk >= end) break;
    float g[2][4], m[2][4], v[2][4];
    uint32_t mc[2], vc[2];
    int64_t e[2];
    int n[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      e[h] = blk * kBlock + 128 * h + 4 * lane;
      const int64_t left = a.n - e[h];
      n[h] = left < 4 ? (left < 0 ? 0 : (int)left) : 4;
      load4(static_cast<const G*>(a.grad), e[h], n[h], g[h]);
      if (E4M3) {
        mc[h] = load_codes(static_cast<const uint8_t*>(a.m), e[h], n[h]);
        vc[h] = load_codes(static_cast<const uint8_t*>(a.v), e[h], n[h]);
      } else {
        load4(static_cast<const float*>(a.m), e[h], n[h], m[h]);
        load4(static_cast<const float*>(a.v), e[h], n[h], v[h]);
      }
    }
    float ms = 0.0f, vs = 0.0f;
    if (E4M3) ms = a.m_scale[blk], vs = a.v_scale[blk];
    float mtop = 0.0f, rtop = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (E4M3) {
        decode4(mc[h], ms, m[h]);
        decode4(vc[h], vs, v[h]);
      }
      // p is fetched here, behind the flat loads of both halves
      float w[4], keep[4];
      Weights<P> at = {};
      const bool any = n[h] > 0;
      bool whole = false;
      if (any) {
        at = find<P>(a, t, e[h]);
        whole = at.n == 4;
        if (MASTER) {
          load4(a.master, e[h], n[h], w);
        } else if (whole) {
          if (((uintptr_t)at.p & (4 * sizeof(P) - 1)) == 0) {
            load4(at.p, 0, 4, w);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = (float)at.p[j];
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) keep[j] = at.keep;
      P* q[4];
      if (any && !whole) {          // a tensor ends here: element by element
        int tj = at.t;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (j < n[h]) {
            const Weights<P> x = find<P>(a, tj, e[h] + j);
            tj = x.t;
            q[j] = x.p;
            keep[j] = x.keep;
            if (!MASTER) w[j] = (float)*x.p;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float gj = __fmul_rn(g[h][j], clip);
        const float old = E4M3 ? __fmul_rn(v[h][j], v[h][j]) : v[h][j];
        m[h][j] = __fadd_rn(__fmul_rn(m[h][j], a.b1), __fmul_rn(gj, a.one_b1));
        const float vj = __fadd_rn(__fmul_rn(old, a.b2), __fmul_rn(__fmul_rn(gj, gj), a.one_b2));
        const float r = __fsqrt_rn(vj);
        v[h][j] = E4M3 ? r : vj;
        if (E4M3) {
          mtop = fmaxf(mtop, fabsf(m[h][j]));
          rtop = fmaxf(rtop, r);
        }
        w[j] = w[j] * keep[j] - __fdividef(m[h][j], r * a.root + a.eps) * a.rate;
      }
      if (any) {
        if (MASTER) store4(a.master, e[h], n[h], w);
        if (whole) {
          if (((uintptr_t)at.p & (4 * sizeof(P) - 1)) == 0) {
            store4(at.p, 0, 4, w);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) at.p[j] = (P)w[j];
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (j < n[h]) *q[j] = (P)w[j];
        }
      }
      if (!E4M3 && any) {
        store4(static_cast<float*>(a.m), e[h], n[h], m[h]);
        store4(static_cast<float*>(a.v), e[h], n[h], v[h]);
      }
    }
    if (E4M3) {
      // largest magnitudes of the block, as bits (they are not negative)
      float mt = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(mtop)));
      float rt = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(rtop)));
      if (mt < 0x1p-100f) mt = 0.0f;
      if (rt < 0x1p-100f) rt = 0.0f;
      const float mi = mt > 0.0f ? __fdiv_rn(448.0f, mt) : 0.0f;
      const float ri = rt > 0.0f ? __fdiv_rn(448.0f, rt) : 0.0f;
      if (lane == 0) {
        a.m_scale[blk] = __fdiv_rn(mt, 448.0f);
        a.v_scale[blk] = __fdiv_rn(rt, 448.0f);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t cm = 0, cr = 0;
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const uint64_t z = mix_word(a.key + (uint64_t)((e[h] + j) / 2 + 1) * kGold);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t u = (uint32_t)(z >> (32 * i));
            const float x = m[h][j + i];
            const uint32_t c = encode(x, mi, u & 0xffffu, false) | (x < 0.0f ? 0x80u : 0u);
            cm |= c << (8 * (j + i));
            cr |= encode(v[h][j + i], ri, u >> 16, true) << (8 * (j + i));
          }
        }
        if (n[h] > 0) {
          store_codes(static_cast<uint8_t*>(a.m), e[h], n[h], cm);
          store_codes(static_cast<uint8_t*>(a.v), e[h], n[h], cr);
        }
      }
    }
  }
}

const void* adamw_fn(int pd, int gd, bool e4m3, bool master) {
#define BKMOO_ADAM(P, G)                                                                    \
  (e4m3 ? (master ? (const void*)adamw_kernel<P, G, true, true>                             \
                  : (const void*)adamw_kernel<P, G, true, false>)                           \
        : (master ? (const void*)adamw_kernel<P, G, false, true>                            \
                  : (const void*)adamw_kernel<P, G, false, false>))
  if (pd == BKMOO_F32) return gd == BKMOO_F32 ? BKMOO_ADAM(float, float) : BKMOO_ADAM(float, __nv_bfloat16);
  return gd == BKMOO_F32 ? BKMOO_ADAM(__nv_bfloat16, float) : BKMOO_ADAM(__nv_bfloat16, __nv_bfloat16);
#undef BKMOO_ADAM
}

// ---- norm ------------------------------------------------------------------

constexpr int kNormThreads = 256;
constexpr int kNormCtas = 1024;      // at most: partial sums in the workspace
static_assert(kNormCtas * sizeof(double) <= BKMOO_NORM_WS_BYTES, "workspace");

// Sum of squares: a thread's in fp32 over 8 vectors at a time, then fp64; a
// CTA's by a fixed tree.  The order is fixed by n alone.
template <class G>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const G* g, int64_t n, double* part) {
  constexpr int V = 16 / sizeof(G);
  const int64_t vecs = n / V, stride = (int64_t)gridDim.x * kNormThreads;
  const uint4* q = reinterpret_cast<const uint4*>(g);
  double sum = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * kNormThreads + threadIdx.x; i < vecs; i += 8 * stride) {
    uint4 x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      x[j] = i + j * stride < vecs ? __ldcs(q + i + j * stride) : make_uint4(0, 0, 0, 0);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (sizeof(G) == 4) {
          const float y = __uint_as_float(w[k]);
          s = fmaf(y, y, s);
        } else {
          const float y = __uint_as_float(w[k] << 16), z = __uint_as_float(w[k] & 0xffff0000u);
          s = fmaf(z, z, fmaf(y, y, s));
        }
      }
    }
    sum += (double)s;
  }
  if (blockIdx.x == 0 && threadIdx.x < n - vecs * V) {
    const float y = (float)g[vecs * V + threadIdx.x];
    sum += (double)(y * y);
  }
  __shared__ double sh[kNormThreads];
  sh[threadIdx.x] = sum;
  __syncthreads();
  for (int w = kNormThreads / 2; w > 0; w >>= 1) {
    if (threadIdx.x < w) sh[threadIdx.x] += sh[threadIdx.x + w];
    __syncthreads();
  }
  if (threadIdx.x == 0) part[blockIdx.x] = sh[0];
}
__global__ void __launch_bounds__(kNormThreads) norm_sum_kernel(const double* part, int n, float* out) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < n; i += kNormThreads) sum += part[i];
  __shared__ double sh[kNormThreads];
  sh[threadIdx.x] = sum;
  __syncthreads();
  for (int w = kNormThreads / 2; w > 0; w >>= 1) {
    if (threadIdx.x < w) sh[threadIdx.x] += sh[threadIdx.x + w];
    __syncthreads();
  }
  if (threadIdx.x == 0) *out = (float)sqrt(sh[0]);
}

bool at(const void* p, uintptr_t by) { return p && ((uintptr_t)p & (by - 1)) == 0; }
bool float_ok(int32_t dt) { return dt == BKMOO_F32 || dt == BKMOO_BF16; }

}  // namespace
}  // namespace bkmoo

using namespace bkmoo;

extern "C" void bkmoo_adamw_default_params(bkmoo_adamw_params* p) {
  if (!p) return;
  p->lr = 1e-3;
  p->beta1 = 0.9;
  p->beta2 = 0.999;
  p->eps = 1e-8;
  p->max_norm = 0.0;
  p->step = 1;
  p->seed = 0;
}

extern "C" int bkmoo_grad_norm(const void* grad, int32_t dtype, int64_t n, float* out_norm, void* ws,
                               size_t ws_bytes, void* stream) {
  if (!float_ok(dtype) || n < 0 || !at(out_norm, 4) || !at(ws, 256) || (n > 0 && !at(grad, 16)))
    return BKMOO_ERR_INVALID;
  if (ws_bytes < BKMOO_NORM_WS_BYTES) return BKMOO_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int64_t per = (int64_t)kNormThreads * 8 * (dtype == BKMOO_F32 ? 4 : 8);
  int64_t ctas = (n + per - 1) / per;
  ctas = ctas < 1 ? 1 : ctas > kNormCtas ? kNormCtas : ctas;
  double* part = static_cast<double*>(ws);
  if (dtype == BKMOO_F32)
    norm_kernel<float><<<(unsigned)ctas, kNormThreads, 0, s>>>(static_cast<const float*>(grad), n, part);
  else
    norm_kernel<__nv_bfloat16><<<(unsigned)ctas, kNormThreads, 0, s>>>(
        static_cast<const __nv_bfloat16*>(grad), n, part);
  norm_sum_kernel<<<1, kNormThreads, 0, s>>>(part, (int)ctas, out_norm);
  return cudaGetLastError() == cudaSuccess ? BKMOO_OK : BKMOO_ERR_CUDA;
}

extern "C" int bkmoo_adamw(void* const* params, const int64_t* sizes, const float* weight_decay,
                           int32_t n_params, int32_t param_dtype, const void* grad,
                           int32_t grad_dtype, float* master, void* m, void* v, float* m_scale,
                           float* v_scale, int32_t state_dtype, const bkmoo_adamw_params* p,
                           const float* grad_norm, void* stream) {
  const bool e4m3 = state_dtype == BKMOO_E4M3;
  if (n_params < 0 || (n_params > 0 && (!params || !sizes)) || !float_ok(param_dtype) ||
      !float_ok(grad_dtype) || (state_dtype != BKMOO_F32 && !e4m3) || !p ||
      (master && param_dtype != BKMOO_BF16))
    return BKMOO_ERR_INVALID;
  if (!(p->beta1 >= 0.0 && p->beta1 < 1.0) || !(p->beta2 >= 0.0 && p->beta2 < 1.0) ||
      !(p->eps >= 0.0) || !std::isfinite(p->lr) || !(p->max_norm >= 0.0) || p->step < 1 ||
      (p->max_norm > 0.0 && !grad_norm) || (grad_norm && !at(grad_norm, 4)))
    return BKMOO_ERR_INVALID;
  const uintptr_t pe = param_dtype == BKMOO_F32 ? 4 : 2;
  int64_t n = 0;
  for (int32_t i = 0; i < n_params; ++i) {
    if (sizes[i] < 0 || (sizes[i] > 0 && !at(params[i], pe)) ||
        (weight_decay && !(weight_decay[i] >= 0.0f && std::isfinite(weight_decay[i]))))
      return BKMOO_ERR_INVALID;
    n += sizes[i];
    if (n > ((int64_t)1 << 42)) return BKMOO_ERR_INVALID;   // one grid holds it
  }
  if (n == 0) return BKMOO_OK;
  if (!at(grad, 16) || !at(m, 16) || !at(v, 16) || (master && !at(master, 16)) ||
      (e4m3 && (!at(m_scale, 4) || !at(v_scale, 4))))
    return BKMOO_ERR_INVALID;
  AdamArgs a;
  a.grad = grad;
  a.m = m;
  a.v = v;
  a.m_scale = m_scale;
  a.v_scale = v_scale;
  a.master = master;
  a.norm = grad_norm;
  a.max_norm = (float)p->max_norm;
  a.b1 = (float)p->beta1;
  a.one_b1 = (float)(1.0 - p->beta1);
  a.b2 = (float)p->beta2;
  a.one_b2 = (float)(1.0 - p->beta2);
  a.rate = (float)(p->lr / (1.0 - std::pow(p->beta1, (double)p->step)));
  a.root = (float)(1.0 / std::sqrt(1.0 - std::pow(p->beta2, (double)p->step)));
  a.eps = (float)p->eps;
  a.key = mix_word(p->seed + ((uint64_t)p->step + 1) * kGold);
  a.n = n;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const void* fn = adamw_fn(param_dtype, grad_dtype, e4m3, master != nullptr);
  // a launch knows kAdamTable tensors; the blocks that lie in them whole are its
  // own, and the next launch begins with the tensor of the first block left
  const int64_t all = (n + kBlock - 1) / kBlock;
  int32_t i = 0;
  int64_t from = 0;            // flat start of tensor i
  for (int64_t first = 0; first < all;) {
    while (sizes[i] == 0 || from + sizes[i] <= first * kBlock) from += sizes[i++];
    int32_t k = 0, j = i;
    int64_t end = from;
    for (; j < n_params && k < kAdamTable; ++j) {
      if (sizes[j] == 0) continue;
      a.p[k] = params[j];
      a.start[k] = end;
      a.keep[k] = (float)(1.0 - p->lr * (double)(weight_decay ? weight_decay[j] : 0.0f));
      end += sizes[j];
      ++k;
    }
    a.start[k] = end;
    a.tensors = k;
    a.first = first;
    a.blocks = (end >= n ? all : end / kBlock) - first;
    void* list[] = {&a};
    if (cudaLaunchKernel(fn, dim3((unsigned)((a.blocks + kAdamSpan - 1) / kAdamSpan)),
                         dim3(kAdamThreads), list, 0, s) != cudaSuccess)
      return BKMOO_ERR_CUDA;
    first += a.blocks;
  }
  return BKMOO_OK;
}
