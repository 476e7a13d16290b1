// What the operators on tokens share (embedding.cu, qk_norm.cu, token_logp.cu): bf16 and
// fp32 elements, whole numbers of 4 or 8 bytes, checks of addresses.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace bkmoo {

inline bool aligned_at(const void* p, uintptr_t by) { return p && ((uintptr_t)p & (by - 1)) == 0; }
inline bool is_float(int32_t dt) { return dt == BKMOO_F32 || dt == BKMOO_BF16; }
inline uintptr_t float_bytes(int32_t dt) { return dt == BKMOO_F32 ? 4 : 2; }
// Whether no two of n arrays of `bytes` overlap.
inline bool apart(const void* const* p, int n, size_t bytes) {
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < i; ++j) {
      const uintptr_t a = (uintptr_t)p[i], b = (uintptr_t)p[j];
      if ((a < b ? b - a : a - b) < bytes) return false;
    }
  return true;
}
inline bool is_id(int32_t bytes) { return bytes == 4 || bytes == 8; }

// (Loads below are plain ones, not by the read-only path: a kernel may begin before the one
// that writes its inputs has ended.)
__device__ __forceinline__ int64_t load_id(const void* ids, int bytes, int64_t i) {
  return bytes == 8 ? static_cast<const int64_t*>(ids)[i] : (int64_t) static_cast<const int32_t*>(ids)[i];
}

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class E>
__device__ __forceinline__ E narrow(float x);
template <>
__device__ __forceinline__ float narrow<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ float2 wide2(uint32_t w) {      // bf16 pair
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint32_t narrow2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Elements of a 16-byte vector.
template <class E>
constexpr int kVec = 16 / (int)sizeof(E);
__device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
  x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = wide2(w[j]);
    x[2 * j] = f.x;
    x[2 * j + 1] = f.y;
  }
}
__device__ __forceinline__ uint4 repack(const float (&x)[4]) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 repack(const float (&x)[8]) {
  return make_uint4(narrow2(x[0], x[1]), narrow2(x[2], x[3]), narrow2(x[4], x[5]), narrow2(x[6], x[7]));
}

}  // namespace bkmoo
