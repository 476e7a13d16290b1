// One AdamW step over all the tensors of a model (include/bkmoo.h), and the norm
// it clips by.
//
// The direction, the moments and the master copy are flat, in the layout of the
// resolve; the weights are tensors of their own.  A warp takes 256 consecutive
// flat elements at a time, whatever tensors they lie in: each lane 4 and 4 more
// 128 further on, so that every access of the flat buffers is a whole vector and
// a warp's accesses are contiguous.  256 is also the block of elements that share
// a scale in 8 bits, so its largest value is a matter of one warp.  The grid
// goes through them side by side.  Which tensor an element belongs to comes from a
// table in the kernel's parameters (one binary search a warp, then steps).
//
// Bound by memory: per element the direction, the weight and both moments (and
// the master copy) are read once and written once.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cmath>
#include <type_traits>

#include "common.cuh"

namespace bkmoo {
namespace {

constexpr int kBlock = 256;          // elements per scale, and per warp and turn
constexpr int kAdamTable = 1024;     // tensors a launch knows
constexpr int kAdamThreads = 256;
constexpr int64_t kAdamWarps = kAdamThreads / 32;

struct AdamArgs {
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;
  float* master;
  const float* norm;                 // or another word that is not finite if there is to be no step
  float max_norm;                    // 0: not clipped
  float b1, one_b1, b2, one_b2;
  float rate;                        // lr / (1 - beta1^step)
  float root;                        // 1 / sqrt(1 - beta2^step)
  float eps;
  float one;                         // 1
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

// Four consecutive elements as they are loaded, and widened to fp32 (8-bit ones
// times their scale).
template <class T>
struct Raw;
template <>
struct Raw<float> {
  float4 x;
};
template <>
struct Raw<__nv_bfloat16> {
  uint2 x;
};
template <>
struct Raw<uint8_t> {
  uint32_t x;
};
template <bool E4M3>
struct State {
  using T = typename std::conditional<E4M3, uint8_t, float>::type;
};

__device__ __forceinline__ Raw<float> load_raw(const float* p) {
  return {__ldcs(reinterpret_cast<const float4*>(p))};
}
__device__ __forceinline__ Raw<__nv_bfloat16> load_raw(const __nv_bfloat16* p) {
  return {__ldcs(reinterpret_cast<const uint2*>(p))};
}
__device__ __forceinline__ Raw<uint8_t> load_raw(const uint8_t* p) {
  return {__ldcs(reinterpret_cast<const uint32_t*>(p))};
}
// The first n of the four, the others 0.
__device__ __forceinline__ Raw<float> load_part(const float* p, int n) {
  return {make_float4(n > 0 ? p[0] : 0.0f, n > 1 ? p[1] : 0.0f, n > 2 ? p[2] : 0.0f, n > 3 ? p[3] : 0.0f)};
}
__device__ __forceinline__ Raw<__nv_bfloat16> load_part(const __nv_bfloat16* p, int n) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = j < n ? __bfloat16_as_ushort(p[j]) : 0u;
  return {make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16)};
}
__device__ __forceinline__ Raw<uint8_t> load_part(const uint8_t* p, int n) {
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < n) w |= (uint32_t)p[j] << (8 * j);
  return {w};
}
__device__ __forceinline__ void widen(const Raw<float>& r, float2 (&x)[2], float) {
  x[0] = make_float2(r.x.x, r.x.y), x[1] = make_float2(r.x.z, r.x.w);
}
__device__ __forceinline__ void widen(const Raw<__nv_bfloat16>& r, float2 (&x)[2], float) {
  x[0] = make_float2(__uint_as_float(r.x.x << 16), __uint_as_float(r.x.x & 0xffff0000u));
  x[1] = make_float2(__uint_as_float(r.x.y << 16), __uint_as_float(r.x.y & 0xffff0000u));
}
__device__ __forceinline__ void widen(const Raw<uint8_t>& r, float2 (&x)[2], float scale) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(r.x >> (16 * j)), __NV_E4M3);
    x[j] = __fmul2_rn(__half22float2(__half2(h)), make_float2(scale, scale));
  }
}
__device__ __forceinline__ void store4(float* p, const float2 (&x)[2]) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(x[0].x, x[0].y, x[1].x, x[1].y));
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float2 (&x)[2]) {
  const __nv_bfloat162 a = __float22bfloat162_rn(x[0]), b = __float22bfloat162_rn(x[1]);
  __stcs(reinterpret_cast<uint2*>(p),
         make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b)));
}
__device__ __forceinline__ void store_part(float* p, int64_t n, const float2 (&x)[2]) {
  if (n >= 4) {
    store4(p, x);
  } else {
    if (n > 0) p[0] = x[0].x;
    if (n > 1) p[1] = x[0].y;
    if (n > 2) p[2] = x[1].x;
  }
}
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t i, int64_t n, uint32_t w) {
  if (n >= 4) {
    __stcs(reinterpret_cast<uint32_t*>(p + i), w);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[i + j] = (uint8_t)(w >> (8 * j));
  }
}

// Four values / their scale as e4m3 bytes, each rounded away from 0 with the
// chance that its rest gives.  `inv` is 1 / scale, and 2^-120 takes e4m3's
// smallest normal number, 2^-6, to fp32's, 2^-126: the product's bits from the
// 20th on are the code, of subnormal values too, and what is below them is the
// rest, of which the upper 16 bits meet the chance's (all 16 places up: the code
// is the top byte; the block's largest value has an empty rest, so no code is
// passed).  w: a word for each value, the chance in its low half (SIGNED) or its
// high half.  FLOOR: what is not 0 does not become 0.
template <bool SIGNED, bool FLOOR>
__device__ __forceinline__ uint32_t encode4(const float2 (&x)[2], float inv, const uint32_t (&w)[4]) {
  uint32_t s[4];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float2 y = __fmul2_rn(__fmul2_rn(x[j], make_float2(inv, inv)), make_float2(0x1p-120f, 0x1p-120f));
    const uint32_t bits[2] = {__float_as_uint(y.x), __float_as_uint(y.y)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s[2 * j + i] = bits[i] * 16 + __byte_perm(w[2 * j + i], 0, SIGNED ? 0x4104 : 0x4324);
      if (FLOOR && bits[i] != 0) s[2 * j + i] = max(s[2 * j + i], 0x1000000u);
    }
  }
  uint32_t c = __byte_perm(__byte_perm(s[0], s[1], 0x0073), __byte_perm(s[2], s[3], 0x0073), 0x5410);
  if (SIGNED) {
    const uint32_t g = __byte_perm(
        __byte_perm(__float_as_uint(x[0].x), __float_as_uint(x[0].y), 0x0073),
        __byte_perm(__float_as_uint(x[1].x), __float_as_uint(x[1].y), 0x0073), 0x5410);
    c |= g & 0x80808080u;
  }
  return c;
}
// The same for a block with a NaN or an infinity: a NaN stays one.
template <bool SIGNED>
__device__ __noinline__ uint32_t encode4_any(float2 x01, float2 x23, float inv, uint32_t w0, uint32_t w1,
                                             uint32_t w2, uint32_t w3) {
  const float x[4] = {x01.x, x01.y, x23.x, x23.y};
  const uint32_t w[4] = {w0, w1, w2, w3};
  uint32_t c = 0;
  for (int j = 0; j < 4; ++j) {
    const uint32_t bits = __float_as_uint(__fmul_rn(__fmul_rn(fabsf(x[j]), inv), 0x1p-120f));
    uint32_t k = min(((bits >> 4) + (SIGNED ? w[j] & 0xffffu : w[j] >> 16)) >> 16, 0x7eu);
    if (!SIGNED) k = max(k, min(bits, 1u));
    if (bits > 0x7f800000u) k = 0x7f;
    if (SIGNED) k |= (__float_as_uint(x[j]) >> 24) & 0x80u;
    c |= k << (8 * j);
  }
  return c;
}

// The tensor of a flat element, from one at or before it on.
__device__ __forceinline__ int tensor_of(const AdamArgs& a, int t, int64_t e) {
  while (t + 1 < a.tensors && a.start[t + 1] <= e) ++t;
  return t;
}

// What a lane has loaded of a block: 4 elements and 4 more 128 further on.
template <class P, class G, bool E4M3>
struct Loaded {
  Raw<G> g[2];
  Raw<typename State<E4M3>::T> m[2], v[2];
  Raw<P> w[2];           // where the weights are read as whole vectors
  float ms, vs;
  P* p;                  // the lane's first weight, NULL: element by element
  float keep;
  int t;                 // the tensor of the block's first element
};

// To 2^-23, of subnormal numbers too.
__device__ __forceinline__ float2 near_root2(float2 x) {
  float2 r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r.x) : "f"(x.x));
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r.y) : "f"(x.y));
  return r;
}
// Rounded root: the hardware's reciprocal root of x, good to 2^-22, and one step of
// Heron's method on x y with the residual in one rounding (x - r r by FMA), which
// leaves an error of 2^-45 before the last rounding: the rounded root but for one in a
// million, in fewer instructions than __fsqrt_rn (4e8 elements 985 us with that).  0 for
// 0, NaN for infinity; not for gradients below 1e-19, whose squares are no normal numbers.
__device__ __forceinline__ float2 root2(float2 x) {
  float2 y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(x.x, 0x1p-126f)));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(x.y, 0x1p-126f)));
  const float2 r = __fmul2_rn(x, y);
  const float2 e = __ffma2_rn(make_float2(-r.x, -r.y), r, x);
  return __ffma2_rn(e, __fmul2_rn(y, make_float2(0.5f, 0.5f)), r);
}
// To 2^-23.
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Two elements' step: moments in place (v as its root in 8 bits), the new weights
// returned.  The moments round as written, product by product, and in 8 bits the root
// is the rounded one: a last bit can move a code, and a code in this step the scale
// of its block in the next.
template <bool E4M3>
struct Step {
  float b1, one_b1, b2, one_b2, rate, root, eps, one, clip;
  __device__ __forceinline__ float2 operator()(float2 g, float2 keep, float2 w, float2& m, float2& v) const {
    auto both = [](float x) { return make_float2(x, x); };
    const float2 gj = __fmul2_rn(g, both(clip));
    const float2 old = E4M3 ? __fmul2_rn(v, v) : v;
    // sums as x 1 + y with a 1 that the compiler does not know: it makes one rounding
    // of a packed product and the sum it goes into
    m = __ffma2_rn(__fmul2_rn(m, both(b1)), both(one), __fmul2_rn(gj, both(one_b1)));
    const float2 vj = __ffma2_rn(__fmul2_rn(old, both(b2)), both(one),
                                 __fmul2_rn(__fmul2_rn(gj, gj), both(one_b2)));
    const float2 r = E4M3 ? root2(vj) : near_root2(vj);
    v = E4M3 ? r : vj;
    const float2 den = __ffma2_rn(r, both(root), both(eps));
    const float2 q = make_float2(reciprocal(den.x), reciprocal(den.y));
    return __ffma2_rn(__fmul2_rn(m, both(-rate)), q, __fmul2_rn(w, keep));
  }
};
__device__ __forceinline__ uint32_t top_of(uint32_t t, float a, float b) {
  return __vimax3_u32(t, __float_as_uint(a) & 0x7fffffffu, __float_as_uint(b) & 0x7fffffffu);
}

template <class P, class G, bool E4M3, bool MASTER>
__global__ void __launch_bounds__(kAdamThreads, 3)
    adamw_kernel(const __grid_constant__ AdamArgs a) {
  grid_wait();
  using S = typename State<E4M3>::T;
  using W = typename std::conditional<MASTER, float, P>::type;    // what the step reads
  const int lane = threadIdx.x & 31;
  const int64_t end = a.first + a.blocks, stride = (int64_t)gridDim.x * kAdamWarps;
  int64_t blk = a.first + (int64_t)blockIdx.x * kAdamWarps + (threadIdx.x >> 5);
  if (blk >= end) return;
  Step<E4M3> step = {a.b1, a.one_b1, a.b2, a.one_b2, a.rate, a.root, a.eps, a.one, a.one};
  if (a.norm) {
    const float norm = *a.norm;
    if (!(fabsf(norm) <= 3.4028235e38f)) return;      // not a step to take
    if (a.max_norm > 0.0f) step.clip = fminf(1.0f, __fdiv_rn(a.max_norm, __fadd_rn(norm, 1e-6f)));
  }
  int t = 0;                        // the tensor of the block's first element
  for (int hi = a.tensors; hi - t > 1;) {
    const int mid = (t + hi) >> 1;
    if (a.start[mid] <= blk * kBlock) t = mid;
    else hi = mid;
  }
  // of that tensor: its end, where its weight 0 of the flat buffers would lie, and
  // whether whole vectors of it are aligned
  int64_t stop = 0;
  P* base = nullptr;
  float keep = 0.0f;
  bool straight = false;
  auto enter = [&](int tensor) {
    t = tensor;
    stop = a.start[t + 1];
    base = static_cast<P*>(a.p[t]) - a.start[t];
    keep = a.keep[t];
    straight = ((uintptr_t)base & (4 * sizeof(P) - 1)) == 0;
  };
  enter(t);

  // Everything of a block that can be loaded at once.
  auto load = [&](int64_t b, Loaded<W, G, E4M3>& x) {
    const int64_t e0 = b * kBlock, e = e0 + 4 * lane;
    if (e0 >= stop) enter(tensor_of(a, t, e0));
    x.t = t;
    x.keep = keep;
    x.p = straight && e0 + kBlock <= stop ? reinterpret_cast<W*>(base + e) : nullptr;
    if (E4M3) x.ms = __ldcs(a.m_scale + b), x.vs = __ldcs(a.v_scale + b);
    if (e0 + kBlock <= a.n) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        x.g[h] = load_raw(static_cast<const G*>(a.grad) + e + 128 * h);
        x.m[h] = load_raw(static_cast<const S*>(a.m) + e + 128 * h);
        x.v[h] = load_raw(static_cast<const S*>(a.v) + e + 128 * h);
        if (MASTER) x.w[h] = load_raw(reinterpret_cast<const W*>(a.master) + e + 128 * h);
        else if (x.p) x.w[h] = load_raw(x.p + 128 * h);
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t left = a.n - (e + 128 * h);
        const int n = left < 4 ? (left < 0 ? 0 : (int)left) : 4;
        x.g[h] = load_part(static_cast<const G*>(a.grad) + e + 128 * h, n);
        x.m[h] = load_part(static_cast<const S*>(a.m) + e + 128 * h, n);
        x.v[h] = load_part(static_cast<const S*>(a.v) + e + 128 * h, n);
        if (MASTER) x.w[h] = load_part(reinterpret_cast<const W*>(a.master) + e + 128 * h, n);
      }
    }
  };

  // 8-bit moments are little data for the work: the next block is fetched ahead
  // of the present one's step.  32-bit ones fill the memory pipe without.
  constexpr bool AHEAD = E4M3;
  // 64-bit words of the lane's pairs of elements: 0 and 1, 64 and 65 from here
  uint64_t word = E4M3 ? a.key + (uint64_t)(blk * (kBlock / 2) + 2 * lane + 1) * kGold : 0;
  const uint64_t word_step = (uint64_t)(stride * (kBlock / 2)) * kGold;
  Loaded<W, G, E4M3> x;
  load(blk, x);
  for (;;) {
    const int64_t next = blk + stride;
    Loaded<W, G, E4M3> y;
    if (AHEAD && next < end) load(next, y);
    const int64_t e = blk * kBlock + 4 * lane;
    float2 m[2][2], v[2][2];
    uint32_t mtop = 0, rtop = 0, rlow = 0xffffffffu;
    if (x.p) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float2 g[2], w[2];
        widen(x.g[h], g, 1.0f);
        widen(x.m[h], m[h], x.ms);
        widen(x.v[h], v[h], x.vs);
        widen(x.w[h], w, 1.0f);
#pragma unroll
        for (int j = 0; j < 2; ++j)
          w[j] = step(g[j], make_float2(x.keep, x.keep), w[j], m[h][j], v[h][j]);
        if (MASTER) {
          store4(a.master + e + 128 * h, w);
          store4(static_cast<P*>(a.p[x.t]) + (e - a.start[x.t]) + 128 * h, w);
        } else {
          store4(reinterpret_cast<P*>(x.p) + 128 * h, w);
        }
      }
    } else {
      // a tensor ends in the block, or its weights lie askew: one by one
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float2 g[2], w[2] = {};
        widen(x.g[h], g, 1.0f);
        widen(x.m[h], m[h], x.ms);
        widen(x.v[h], v[h], x.vs);
        if (MASTER) widen(x.w[h], w, 1.0f);
        P* p[4] = {};
        float keeps[4] = {};
        int tj = x.t;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int64_t i = e + 128 * h + j;
          if (i < a.n) {
            tj = tensor_of(a, tj, i);
            p[j] = static_cast<P*>(a.p[tj]) + (i - a.start[tj]);
            keeps[j] = a.keep[tj];
            if (!MASTER) (j & 1 ? w[j / 2].y : w[j / 2].x) = (float)*p[j];
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float2 m2 = m[h][j], v2 = v[h][j];
          w[j] = step(g[j], make_float2(keeps[2 * j], keeps[2 * j + 1]), w[j], m2, v2);
          if (p[2 * j]) {
            *p[2 * j] = (P)w[j].x;
            if (MASTER) a.master[e + 128 * h + 2 * j] = w[j].x;
            m[h][j].x = m2.x, v[h][j].x = v2.x;
          }
          if (p[2 * j + 1]) {
            *p[2 * j + 1] = (P)w[j].y;
            if (MASTER) a.master[e + 128 * h + 2 * j + 1] = w[j].y;
            m[h][j].y = m2.y, v[h][j].y = v2.y;
          }
        }
      }
    }
    const int64_t left = a.n - e;
    if (E4M3) {
      // largest magnitudes of the block, as bits (a NaN is above all)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          mtop = top_of(mtop, m[h][j].x, m[h][j].y);
          rtop = __vimax3_u32(rtop, __float_as_uint(v[h][j].x), __float_as_uint(v[h][j].y));
          rlow = __vimin3_u32(rlow, __float_as_uint(v[h][j].x), __float_as_uint(v[h][j].y));
        }
      mtop = __reduce_max_sync(0xffffffffu, mtop);
      rtop = __reduce_max_sync(0xffffffffu, rtop);
      rlow = __reduce_min_sync(0xffffffffu, rlow);
      if (mtop < 0x0d800000u) mtop = 0;               // below 2^-100
      if (rtop < 0x0d800000u) rtop = 0;
      const float mt = __uint_as_float(mtop), rt = __uint_as_float(rtop);
      const float each = __frcp_rn((lane & 1) ? rt : mt);       // both reciprocals at once
      const float mi = mtop != 0 ? __fmul_rn(448.0f, __shfl_sync(0xffffffffu, each, 0)) : 0.0f;
      const float ri = rtop != 0 ? __fmul_rn(448.0f, __shfl_sync(0xffffffffu, each, 1)) : 0.0f;
      if (lane == 0) a.m_scale[blk] = __fmul_rn(mt, 1.0f / 448.0f);
      if (lane == 1) a.v_scale[blk] = __fmul_rn(rt, 1.0f / 448.0f);
      const bool plain = mtop < 0x7f800000u && rtop < 0x7f800000u;
      // no root is as small as a code of 0
      const bool above = __float_as_uint(__uint_as_float(rlow) * ri * 0x1p-120f) >= 0x100000u;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t u[4], cm, cr;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint64_t z = mix_word(word + (uint64_t)(64 * h + j) * kGold);
          u[2 * j] = (uint32_t)z;
          u[2 * j + 1] = (uint32_t)(z >> 32);
        }
        if (plain) {
          cm = encode4<true, false>(m[h], mi, u);
          cr = above ? encode4<false, false>(v[h], ri, u) : encode4<false, true>(v[h], ri, u);
        } else {
          cm = encode4_any<true>(m[h][0], m[h][1], mi, u[0], u[1], u[2], u[3]);
          cr = encode4_any<false>(v[h][0], v[h][1], ri, u[0], u[1], u[2], u[3]);
        }
        store_codes(static_cast<uint8_t*>(a.m), e + 128 * h, left - 128 * h, cm);
        store_codes(static_cast<uint8_t*>(a.v), e + 128 * h, left - 128 * h, cr);
      }
      word += word_step;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        store_part(static_cast<float*>(a.m) + e + 128 * h, left - 128 * h, m[h]);
        store_part(static_cast<float*>(a.v) + e + 128 * h, left - 128 * h, v[h]);
      }
    }
    if (next >= end) break;
    blk = next;
    if (AHEAD) x = y;
    else load(blk, x);
  }
}

// A master copy goes with bf16 weights.
template <class G, bool E4M3>
const void* adamw_fn(bool f32_params, bool master) {
  if (f32_params) return (const void*)adamw_kernel<float, G, E4M3, false>;
  return master ? (const void*)adamw_kernel<__nv_bfloat16, G, E4M3, true>
                : (const void*)adamw_kernel<__nv_bfloat16, G, E4M3, false>;
}
const void* adamw_fn(int pd, int gd, bool e4m3, bool master) {
  const bool f = pd == BKMOO_F32;
  if (gd == BKMOO_F32) return e4m3 ? adamw_fn<float, true>(f, master) : adamw_fn<float, false>(f, master);
  return e4m3 ? adamw_fn<__nv_bfloat16, true>(f, master) : adamw_fn<__nv_bfloat16, false>(f, master);
}

// ---- norm ------------------------------------------------------------------

constexpr int kNormThreads = 256;
// At most, four an SM, so that one wave holds them: 4e8 bf16 137 us, 5.8 TB/s (1024,
// of which 912 fit at a time, 162).
constexpr int kNormCtas = 608;
static_assert(kNormCtas * sizeof(double) <= BKMOO_NORM_WS_BYTES, "workspace");

// Sum of squares: a thread's in fp32 over 8 vectors at a time, then fp64; a
// CTA's by a fixed tree.  The order is fixed by n alone.  (64 squares of bf16 values
// come out 4e-8 of them low, for ties are frequent there: half a rounding of the fp32
// result.  Four at a time with the roundings kept beside, 185 us for 4e8 elements
// instead of 137.)
template <class G>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const G* g, int64_t n, double* part) {
  grid_wait();
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
    sum += (double)y * (double)y;
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
// `gave_up`: NULL, or what makes the norm of a gradient that may be undefined NaN.
__global__ void __launch_bounds__(kNormThreads)
    norm_sum_kernel(const double* part, int n, float* out, const float* gave_up) {
  grid_wait();
  double sum = 0.0;
  for (int i = threadIdx.x; i < n; i += kNormThreads) sum += part[i];
  __shared__ double sh[kNormThreads];
  sh[threadIdx.x] = sum;
  __syncthreads();
  for (int w = kNormThreads / 2; w > 0; w >>= 1) {
    if (threadIdx.x < w) sh[threadIdx.x] += sh[threadIdx.x + w];
    __syncthreads();
  }
  if (threadIdx.x == 0) *out = __fsqrt_rn((float)sh[0]) + (gave_up ? *gave_up : 0.0f);
}

// The device's word that is 0, or NaN once a tile kernel has given up; NULL where no such
// kernel can have run yet (the first call on a device, during a capture).
const float* gave_up_word(cudaStream_t s) {
  int32_t* word = nullptr;
  return tile_status_word(s, &word) == BKMOO_OK ? reinterpret_cast<const float*>(word + 1) : nullptr;
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
  int parts = (int)ctas;
  void* first[] = {&grad, &n, &part};
  const float* gave_up = gave_up_word(s);
  void* second[] = {&part, &parts, &out_norm, &gave_up};
  const void* fn = dtype == BKMOO_F32 ? (const void*)norm_kernel<float>
                                      : (const void*)norm_kernel<__nv_bfloat16>;
  if (launch_behind(fn, dim3(parts), dim3(kNormThreads), first, 0, s, true) != cudaSuccess ||
      launch_behind((const void*)norm_sum_kernel, dim3(1), dim3(kNormThreads), second, 0, s, true) !=
          cudaSuccess)
    return BKMOO_ERR_CUDA;
  return BKMOO_OK;
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
    if (n > ((int64_t)1 << 48)) return BKMOO_ERR_INVALID;
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
  a.one = 1.0f;
  a.key = mix_word(p->seed + ((uint64_t)p->step + 1) * kGold);
  a.n = n;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // Whether the gradient may be of a tile kernel that gave up: a norm says so itself
  // (norm_sum_kernel), the word that it has it from does without one.  (Looking at both in
  // the kernel spilled registers: 1.2e9 elements of 8-bit moments 3512 us, 3179 so.)
  if (!a.norm) a.norm = gave_up_word(s);
  const void* fn = adamw_fn(param_dtype, grad_dtype, e4m3, master != nullptr);
  int dev = 0, sms = 0, per_sm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, fn, kAdamThreads, 0) != cudaSuccess)
    return BKMOO_ERR_CUDA;
  const int64_t grid = (int64_t)sms * (per_sm < 1 ? 1 : per_sm);
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
    int64_t ctas = (a.blocks + kAdamWarps - 1) / kAdamWarps;
    if (ctas > grid) ctas = grid;
    void* list[] = {&a};
    if (launch_behind(fn, dim3((unsigned)ctas), dim3(kAdamThreads), list, 0, s, true) != cudaSuccess)
      return BKMOO_ERR_CUDA;
    first += a.blocks;
  }
  return BKMOO_OK;
}
