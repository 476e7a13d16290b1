// The matrix products of the gated projections and of the per-language weight
// gradients, on the tensor cores: one persistent kernel in three kinds.
//
//   kGate    [a | b] = x [Wg; Wu]^T, h = act(a) b       sum over the input width
//   kInput   dx = da Wg + db Wu                         sum over the hidden width
//   kWeight  dW_k = dy_k^T x_k for every language k     sum over its rows
//   kBoth    a launch of kInput's tiles and then kWeight's: the few long ones first,
//            the many short ones where SMs come free
//
// A tile is 128 rows (256 with a CTA pair) by BN = 64, 128 or 256 columns of fp32
// accumulators; for kGate half of them columns of a and half the same ones of b, so
// that h is formed where both are.  Warp 8 of a CTA copies operand tiles of 64 along the sum into a
// ring of stages (TMA, 128-byte swizzle, rows and columns beyond the matrix are
// zeros), one thread of warp 9 issues the products (tcgen05) into one of two
// accumulators in tensor memory, and warps 0-7 take the other to global memory
// meanwhile.  Operands whose sum runs across their rows (kInput's W, kWeight's
// dy and x) are read as they lie: the products take them across, no transposed
// copy is made.  All sums are fp32; a result is rounded once, when it is stored.
#pragma once

#include <cuda_bf16.h>

#include <type_traits>

#include "tensor_core.cuh"

namespace bkmoo {

// How kWeight's results are written, a kernel each (one for all spills registers, 3.5 %
// of the plain one's time and more of the others'): bf16 in whole aligned pieces; bf16
// added to what is there, the same; bf16 in pieces that are not whole or not aligned,
// added or not; fp32, whole and aligned or not, and each of them added or not.
enum TileMode {
  kPlain = 0, kAdded = 1, kTurned = 2, kSums = 3, kSumsTurned = 4, kSumsAdded = 5, kSumsTurnedAdded = 6
};
constexpr bool mode_f32(int mode) { return mode >= kSums; }
constexpr bool mode_turned(int mode) {
  return mode == kTurned || mode == kSumsTurned || mode == kSumsTurnedAdded;
}
// Kernels that fetch ahead what they add to (fetch_tile).
constexpr bool mode_ahead(int mode) {
  return mode == kAdded || mode == kSumsAdded || mode == kSumsTurnedAdded;
}
enum TileKind { kGate = 0, kInput = 1, kWeight = 2, kBoth = 3 };

constexpr int kTileM = 128;    // rows of a CTA's tile
constexpr int kTileK = 64;     // of the sum per stage: 128 bytes, the swizzle's row
constexpr int kTileEpilogueWarps = 8;
constexpr int kTileThreads = 32 * (kTileEpilogueWarps + 2);
constexpr int kTileGroupM = 8;  // tiles of rows that are worked on together

// cg: CTAs that share a tile, bn: its columns.
__host__ __device__ constexpr int tile_stage_bytes(int cg, int bn) {
  return (kTileM + bn / cg) * kTileK * 2;
}
__host__ __device__ constexpr int tile_stages(int cg, int bn) {
  return 196608 / tile_stage_bytes(cg, bn);
}
// Where a warp turns 32 x 32 results from rows of lanes to rows of memory.
constexpr int kTurnBytes = 32 * 33 * 4;
__host__ __device__ constexpr int tile_smem(int cg, int bn) {
  return tile_stages(cg, bn) * tile_stage_bytes(cg, bn) + 1024 +   // stages start on 1024 bytes
         kTileEpilogueWarps * kTurnBytes;
}

// Where a result goes: rows of `ld` elements.  `vec` is the widest store that every
// row's 32-column pieces allow: 32 or 16 bytes, and for kWeight also 4 or 0 (no more
// than an element).
struct TileOut {
  void* p;
  int64_t ld;
  int32_t vec;
};

template <int KIND>
struct TileArgs;

template <>
struct TileArgs<kGate> {
  CUtensorMap a, b[2];          // x; Wg, Wu
  TileOut out[3];               // h, a, b; p = NULL: not wanted
  int32_t* status;
  int32_t rows, cols;           // T, F
  int32_t tiles_m, tiles_n, tiles;
  int32_t nkt;
  int32_t act;
  int32_t withhold;             // self-test: no operand is ever copied, every wait runs out
};
template <>
struct TileArgs<kInput> {
  CUtensorMap a[2], b[2];       // da, db; Wg, Wu
  TileOut out;                  // dx
  int32_t rows, cols;           // T, D
  int32_t tiles_m, tiles_n, tiles;
  int32_t nkt;                  // of one of the two products
};
// Up to two matrices dy (da and db) against one x, for every language.  Empty
// languages have no map; their gradient is zero.
template <>
struct TileArgs<kWeight> {
  CUtensorMap a[2 * kMaxK], b[kMaxK];
  void* out[2 * kMaxK];         // [matrix][language], contiguous rows of `cols`
  int32_t vec[2 * kMaxK];
  int32_t nkt[kMaxK];
  int32_t order[kMaxK];         // languages, the longest first
  int32_t* status;
  int32_t rows, cols;
  int32_t tiles_m, tiles_n, tiles;
  int32_t mats, n_lang;
  int32_t out_dtype, accumulate;
};

template <>
struct TileArgs<kBoth> {
  TileArgs<kInput> in;
  TileArgs<kWeight> w;
  int32_t* status;
  int32_t head_start;           // see Walk
};

// The tiles of one CTA or pair: `unit` of `units`, every units-th of the first set
// and then of the second.  Units that get one tile of the first set less than others
// begin with head_start tiles of the second among themselves.
struct Walk {
  int unit, units, a, b, head, more;   // more: units with one tile of the first set more
  int k = 0;
  __device__ __forceinline__ Walk(int unit_, int units_, int a_, int b_, int head_)
      : unit(unit_), units(units_), a(a_), b(b_), more(a_ % units_) {
    head = more ? head_ : 0;
  }
  // The next tile: 0 none left, 1 of the first set, 2 of the second.
  __device__ __forceinline__ int next(int& tile) {
    tile = unit + k * units;
    if (tile < a) {
      ++k;
      return 1;
    }
    const int j = k - a / units - (unit < more ? 1 : 0);   // of the second set
    const bool early = more && unit >= more;
    ++k;
    if (early && j < head) tile = j * (units - more) + unit - more;
    else tile = head * (units - more) + (j - (early ? head : 0)) * units + unit;
    return tile < b ? 2 : 0;
  }
};

struct Tile {
  int g, m0, n0, nkt;   // g: kWeight's matrix * kMaxK + language
  int span;             // steps of the sum that one accumulator takes (kExactSteps)
};
// The tensor cores drop what an addition shifts out of the accumulator: a sum of T
// rows comes out about 1e-9 T of it low (1.9e-5 for 16384, more than all other
// roundings of fp32 products together).  bf16 results do not show it.  For fp32 ones
// an accumulator takes 512 of the sum, 5e-7, and the pieces are added in registers,
// rounded to nearest; tiles are then at most 128 columns wide, for the registers.
constexpr int kExactSteps = 8;

template <int KIND, int CG, int BN>
__device__ __forceinline__ Tile tile_at(const TileArgs<KIND>& p, int t) {
  Tile r;
  int i = t;
  r.g = 0;
  r.span = 1 << 30;
  if constexpr (KIND == kWeight) {
    if (p.out_dtype == BKMOO_F32) r.span = kExactSteps;
    const int per = p.tiles_m * p.tiles_n;
    const int unit = t / per;                 // language by language, its matrices in turn
    i = t - unit * per;
    const int lang = p.order[unit / p.mats];
    r.g = (unit % p.mats) * kMaxK + lang;
    r.nkt = p.nkt[lang];
  } else if constexpr (KIND == kInput) {
    r.nkt = 2 * p.nkt;
  } else {
    r.nkt = p.nkt;
  }
  // kTileGroupM tiles of rows at a time, so that the tiles in flight share both
  // their rows' and their columns' operands in L2
  const int band = kTileGroupM * p.tiles_n, b = i / band;
  const int first = b * kTileGroupM;
  const int high = p.tiles_m - first < kTileGroupM ? p.tiles_m - first : kTileGroupM;
  const int j = i - b * band;
  r.m0 = (first + j % high) * (kTileM * CG);
  r.n0 = (j / high) * (KIND == kGate ? BN / 2 : BN);
  return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ void st_global32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]),
               "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// 32 columns of one row, the first n of which exist, 16-byte aligned.
__device__ __forceinline__ void store_row(__nv_bfloat16* p, const float (&v)[32], int n, int vec) {
  uint32_t w[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
  if (vec == 32 && n >= 32) {
    st_global32(p, w);
    st_global32(p + 16, w + 8);
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (n >= 8 * j + 8) {
      reinterpret_cast<uint4*>(p)[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (8 * j + i < n) p[8 * j + i] = __float2bfloat16_rn(v[8 * j + i]);
    }
  }
}
// A warp's 32 rows of COLS bf16 columns (w: this lane's row) to memory, of which the
// first `rows` exist, all 16-byte aligned: through shared memory, 16 bytes a lane, so
// that a store covers whole lines (8 or 4 lanes a row) instead of 32 bytes of 32 rows.
// Chunks of 16 bytes lie at their place xor the row's, free of bank conflicts.
template <int COLS>
__device__ __forceinline__ void put_block(__nv_bfloat16* first, int64_t ld, const uint32_t (&w)[COLS / 2],
                                          int rows, float* turn) {
  constexpr int CH = COLS / 8;
  const int lane = threadIdx.x & 31;
  auto place = [](int row, int j) { return row * CH + (j ^ (CH == 8 ? row & 7 : (row >> 1) & 3)); };
  uint4* t = reinterpret_cast<uint4*>(turn);
#pragma unroll
  for (int j = 0; j < CH; ++j)
    t[place(lane, j)] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
  __syncwarp();
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int row = (k * 32 + lane) / CH, j = lane % CH;
    if (row < rows) *reinterpret_cast<uint4*>(first + row * ld + 8 * j) = t[place(row, j)];
  }
  __syncwarp();
}
// The first n columns of one row of them.
template <int W>
__device__ __forceinline__ void put_some(__nv_bfloat16* p, const uint32_t (&w)[W], int n) {
#pragma unroll
  for (int j = 0; j < W / 4; ++j) {
    if (n >= 8 * j + 8) {
      reinterpret_cast<uint4*>(p)[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (8 * j + i < n)
          p[8 * j + i] = __ushort_as_bfloat16((unsigned short)(w[4 * j + i / 2] >> (16 * (i & 1))));
    }
  }
}
// The same of 32 fp32 columns, rounded to T and added to what is there where `add`.
__device__ __forceinline__ void put4(float* q, float4 x, bool add, float4 old) {
  if (add) x.x += old.x, x.y += old.y, x.z += old.z, x.w += old.w;
  *reinterpret_cast<float4*>(q) = x;
}
__device__ __forceinline__ void put4(__nv_bfloat16* q, float4 x, bool add, uint2 old) {
  if (add) {
    x.x += __uint_as_float(old.x << 16), x.y += __uint_as_float(old.x & 0xffff0000u);
    x.z += __uint_as_float(old.y << 16), x.w += __uint_as_float(old.y & 0xffff0000u);
  }
  *reinterpret_cast<uint2*>(q) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
}
template <class T>
__device__ __forceinline__ void put_sums(T* first, int64_t ld, const float (&v)[32], int rows, bool add,
                                         float* turn) {
  using Four = typename std::conditional<sizeof(T) == 4, float4, uint2>::type;
  const int lane = threadIdx.x & 31, j = lane & 7;
  float4* t = reinterpret_cast<float4*>(turn);
  T* q = first + (lane >> 3) * ld + 4 * j;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    t[lane * 8 + (i ^ (lane & 7))] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  __syncwarp();
  Four old[8];
  if (add) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (4 * k + (lane >> 3) < rows) old[k] = *reinterpret_cast<const Four*>(q + 4 * k * ld);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int row = 4 * k + (lane >> 3);
    if (row < rows) put4(q + 4 * k * ld, t[row * 8 + (j ^ (row & 7))], add, old[k]);
  }
  __syncwarp();
}
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void as_type(float* p, float x) { *p = x; }
__device__ __forceinline__ void as_type(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// The warp's 32 rows of 32 columns, of which the first `rows` and n exist, where they
// are not aligned for wide vectors: turned in shared memory (turn: rows of 33 floats,
// of which 32 are the piece's), so that the warp writes a row at a time, 32
// neighbours, instead of one element of 32 rows.  What they are added to is fetched 16
// rows at a time.
template <class T>
__device__ __forceinline__ void put_turned(T* p, int64_t ld, int rows, int n, bool add, const float* turn) {
  const int lane = threadIdx.x & 31, here = lane < n ? rows : 0;
  T* q = p + lane;
  turn += lane;
#pragma unroll 1
  for (int r0 = 0; r0 < 32; r0 += 16, q += 16 * ld, turn += 16 * 33) {
    T old[16];
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (add && r0 + r < here) old[r] = q[r * ld];
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (r0 + r < here) as_type(q + r * ld, add ? turn[r * 33] + as_float(old[r]) : turn[r * 33]);
  }
}
// bf16 by pairs (4-byte aligned, ld and so n even): two rows at a time, the upper
// lanes the second.
__device__ __forceinline__ void put_turned_pairs(__nv_bfloat16* p, int64_t ld, int rows, int n, bool add,
                                                 const float* turn) {
  const int lane = threadIdx.x & 31, up = lane >> 4, c = 2 * (lane & 15), here = c < n ? rows - up : 0;
  uint32_t* q = reinterpret_cast<uint32_t*>(p + up * ld + c);
  turn += up * 33 + c;
#pragma unroll 1
  for (int r0 = 0; r0 < 32; r0 += 16, q += 8 * ld, turn += 16 * 33) {
    uint32_t old[8];
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (add && r0 + 2 * r < here) old[r] = q[r * ld];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      if (r0 + 2 * r < here) {
        float lo = turn[r * 66], hi = turn[r * 66 + 1];
        if (add) lo += __uint_as_float(old[r] << 16), hi += __uint_as_float(old[r] & 0xffff0000u);
        q[r * ld] = pack_bf16(lo, hi);
      }
    }
  }
}

__device__ __forceinline__ void store_bf16(const TileOut& o, int64_t row, int col,
                                           const float (&v)[32], int n) {
  if (o.p) store_row(static_cast<__nv_bfloat16*>(o.p) + row * o.ld + col, v, n, o.vec);
}

// ---- activations, two values at a time ---------------------------------------
//
// silu a s with s = 1 / (1 + e^-a); gelu_tanh a s with s = 1 / (1 + e^(-2 z)), z =
// sqrt(2/pi) (a + 0.044715 a^3), which is a (1 + tanh z) / 2 without its
// cancellation; gelu a Phi(a) with Phi(a) = erfc(-a / sqrt 2) / 2 and erfc by the
// Chebyshev fit of Numerical Recipes (section 6.2: erfc(x) = t e^(-x^2 + P(t)) for
// x >= 0, t = 1 / (1 + x / 2), fractional error below 1.2e-7), e^(-x^2) of which is
// the derivative's too.  Powers of 2 and reciprocals are the hardware's, good to
// about 2^-22 and rounded arguments' worth more: 2^-18 at most.  Where e^-a, or the bell
// of gelu, leaves fp32's normal numbers (a < -87 and -13) the result, below 1e-35 there,
// is 0.
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 power2(float2 x) {
  float2 r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(x.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(x.y));
  return r;
}
__device__ __forceinline__ float2 inverse(float2 x) {
  float2 r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(x.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(x.y));
  return r;
}
// 1 / (1 + 2^-x)
__device__ __forceinline__ float2 sigmoid2(float2 x) {
  return inverse(__fadd2_rn(power2(make_float2(-x.x, -x.y)), both(1.0f)));
}
// Phi(a), and e^(-a^2 / 2).
__device__ __forceinline__ float2 normal2(float2 a, float2* bell) {
  constexpr float kLog2e = 1.44269504f;
  const float2 x = __fmul2_rn(make_float2(fabsf(a.x), fabsf(a.y)), both(0.70710678f));
  const float2 t = inverse(__ffma2_rn(x, both(0.5f), both(1.0f)));
  float2 q = both(0.17087277f);
  q = __ffma2_rn(q, t, both(-0.82215223f));
  q = __ffma2_rn(q, t, both(1.48851587f));
  q = __ffma2_rn(q, t, both(-1.13520398f));
  q = __ffma2_rn(q, t, both(0.27886807f));
  q = __ffma2_rn(q, t, both(-0.18628806f));
  q = __ffma2_rn(q, t, both(0.09678418f));
  q = __ffma2_rn(q, t, both(0.37409196f));
  q = __ffma2_rn(q, t, both(1.00002368f));
  q = __ffma2_rn(q, t, both(-1.26551223f));
  const float2 e = power2(__fmul2_rn(__fmul2_rn(a, a), both(-0.5f * kLog2e)));
  *bell = e;
  // half of erfc(|x|): Phi on the negative side
  const float2 low = __fmul2_rn(__fmul2_rn(__fmul2_rn(t, both(0.5f)), e), power2(__fmul2_rn(q, both(kLog2e))));
  return make_float2(a.x < 0.0f ? low.x : 1.0f - low.x, a.y < 0.0f ? low.y : 1.0f - low.y);
}
// 2 z of gelu_tanh times log2(e), and its derivative by a without the factor log2(e).
__device__ __forceinline__ float2 tanh_arg(float2 a, float2 q) {
  constexpr float k = 1.59576912f * 1.44269504f;
  return __fmul2_rn(__fmul2_rn(a, both(k)), __ffma2_rn(q, both(0.044715f), both(1.0f)));
}
__device__ __forceinline__ float2 activation2(int act, float2 a) {
  if (act == BKMOO_SILU) return __fmul2_rn(a, sigmoid2(__fmul2_rn(a, both(1.44269504f))));
  if (act == BKMOO_GELU) {
    float2 bell;
    return __fmul2_rn(a, normal2(a, &bell));
  }
  return __fmul2_rn(a, sigmoid2(tanh_arg(a, __fmul2_rn(a, a))));
}
// act(a) and act'(a).
__device__ __forceinline__ void activation_slope2(int act, float2 a, float2* f, float2* df) {
  if (act == BKMOO_SILU) {
    const float2 s = sigmoid2(__fmul2_rn(a, both(1.44269504f)));
    *f = __fmul2_rn(a, s);
    *df = __ffma2_rn(*f, __ffma2_rn(s, both(-1.0f), both(1.0f)), s);
  } else if (act == BKMOO_GELU) {
    float2 bell;
    const float2 c = normal2(a, &bell);
    *f = __fmul2_rn(a, c);
    *df = __ffma2_rn(__fmul2_rn(a, both(0.39894228f)), bell, c);
  } else {
    const float2 q = __fmul2_rn(a, a), s = sigmoid2(tanh_arg(a, q));
    *f = __fmul2_rn(a, s);
    // (a finite dz, for where a^2 is not its factor is 0)
    const float2 dz = __ffma2_rn(make_float2(fminf(q.x, 1e30f), fminf(q.y, 1e30f)),
                                 both(3.0f * 0.044715f * 1.59576912f), both(1.59576912f));
    *df = __ffma2_rn(__fmul2_rn(*f, __ffma2_rn(s, both(-1.0f), both(1.0f))), dz, s);
  }
}
__device__ __forceinline__ float activation(int act, float a) { return activation2(act, both(a)).x; }
__device__ __forceinline__ void activation_slope(int act, float a, float* f, float* df) {
  float2 f2, d2;
  activation_slope2(act, both(a), &f2, &d2);
  *f = f2.x;
  *df = d2.x;
}

template <int CG, int BN>
struct TileShared {
  uint64_t full[tile_stages(CG, BN)], empty[tile_stages(CG, BN)];  // full: the first CTA's, for both
  uint64_t tfull[2], tempty[2];                                    // tempty: the first CTA's, for both
  uint64_t drain;
  uint32_t tmem;
  volatile int abort;
};

// Operand tiles of one step of the sum.
template <int KIND, int CG, int BN>
__device__ __forceinline__ void load_step(const TileArgs<KIND>& p, const Tile& t, int kt,
                                          unsigned rank, unsigned char* a, unsigned char* b,
                                          uint32_t bar) {
  const int m = t.m0 + (int)rank * kTileM;
  if constexpr (KIND == kGate) {
    tile_load<CG>(a, &p.a, kt * kTileK, m, bar);
    if (CG == 1) {
      tile_load<CG>(b, &p.b[0], kt * kTileK, t.n0, bar);
      tile_load<CG>(b + BN / 2 * kTileK * 2, &p.b[1], kt * kTileK, t.n0, bar);
    } else {
      tile_load<CG>(b, &p.b[rank], kt * kTileK, t.n0, bar);
    }
  } else {
    const CUtensorMap* bm;
    int y;
    if constexpr (KIND == kInput) {
      const int second = kt >= p.nkt;
      y = (kt - (second ? p.nkt : 0)) * kTileK;
      tile_load<CG>(a, &p.a[second], y, m, bar);
      bm = &p.b[second];
    } else {
      y = kt * kTileK;
      tile_load<CG>(a, &p.a[t.g], m, y, bar);
      tile_load<CG>(a + 64 * kTileK * 2, &p.a[t.g], m + 64, y, bar);
      bm = &p.b[t.g % kMaxK];
    }
    const int n = t.n0 + (int)rank * (BN / CG);
#pragma unroll
    for (int c = 0; c < BN / CG / 64; ++c)
      tile_load<CG>(b + c * 64 * kTileK * 2, bm, n + 64 * c, y, bar);
  }
}

// A warp's 32 rows (this thread's: `row`) by 32 columns of a gradient.
template <class T, int MODE>
__device__ __forceinline__ void put_piece(const TileArgs<kWeight>& p, const Tile& t, int row, int at,
                                          float (&v)[32], int n, float* turn) {
  const int lane = threadIdx.x & 31, rows = p.rows - (row - lane);
  T* first = static_cast<T*>(p.out[t.g]) + (int64_t)(row - lane) * p.cols + t.n0 + at;
  if (!mode_turned(MODE) || (p.vec[t.g] >= 16 && n >= 32)) {
    put_sums(first, p.cols, v, rows, p.accumulate, turn);
    return;
  }
  if constexpr (mode_turned(MODE)) {
#pragma unroll
    for (int j = 0; j < 32; ++j) turn[lane * 33 + j] = v[j];
    __syncwarp();
    if constexpr (sizeof(T) == 2) {
      if (p.vec[t.g] != 0) put_turned_pairs(first, p.cols, rows, n, p.accumulate, turn);
      else put_turned(first, p.cols, rows, n, p.accumulate, turn);
    } else {
      put_turned(first, p.cols, rows, n, p.accumulate, turn);
    }
    __syncwarp();
  }
}

// One warp's share of a finished tile: rows of its quarter, columns of its half.
// `acc`: the accumulator's tensor-memory address for this warp's lanes; `empty`:
// the tile's sum is empty and the accumulator was not written.
template <int KIND, int BN, int MODE>
__device__ __forceinline__ void take_tile(const TileArgs<KIND>& p, const Tile& t, int row, int half,
                                          uint32_t acc, bool empty, float* turn,
                                          const float (*before)[32]) {
  const bool live = row < p.rows;
  if constexpr (KIND == kGate) {
#pragma unroll 1
    for (int at = 32 * half; at < BN / 2; at += 64) {
      const int n = p.cols - (t.n0 + at);
      uint32_t ra[32], rb[32];
      tc_load32(ra, acc + at);
      tc_load32(rb, acc + BN / 2 + at);
      tc_landed(ra);
      tc_landed(rb);
      if (live && n > 0) {
        float a[32], b[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          a[j] = __uint_as_float(ra[j]);
          b[j] = __uint_as_float(rb[j]);
        }
        store_bf16(p.out[1], row, t.n0 + at, a, n);
        store_bf16(p.out[2], row, t.n0 + at, b, n);
        if (p.out[0].p) {
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float2 f = activation2(p.act, make_float2(a[j], a[j + 1]));
            a[j] = f.x * b[j];
            a[j + 1] = f.y * b[j + 1];
          }
          store_bf16(p.out[0], row, t.n0 + at, a, n);
        }
      }
      __syncwarp();   // the loads are the whole warp's
    }
  } else {
    // the half's columns, in pieces of 32; two at a time where they go out as bf16
    // whole lines
    __nv_bfloat16* block = nullptr;
    int64_t ld = 0;
    if constexpr (KIND == kInput) {
      block = static_cast<__nv_bfloat16*>(p.out.p), ld = p.out.ld;
    } else if constexpr (MODE == kPlain) {
      block = static_cast<__nv_bfloat16*>(p.out[t.g]), ld = p.cols;
    }
    const int row0 = row - (int)(threadIdx.x & 31);
    constexpr int WIDE = BN >= 128 ? 64 : 32;
    if constexpr (KIND == kInput || MODE == kPlain) {
#pragma unroll 1
      for (int c = 0; c < BN / 2; c += WIDE) {
        const int at = half * (BN / 2) + c, n = p.cols - (t.n0 + at);
        if (n <= 0) break;
        uint32_t w[WIDE / 2];
#pragma unroll
        for (int i = 0; i < WIDE / 32; ++i) {
          uint32_t r[32];
          if (!empty) {
            tc_load32(r, acc + at + 32 * i);
            tc_landed(r);
          }
#pragma unroll
          for (int j = 0; j < 16; ++j)
            w[16 * i + j] = empty ? 0u : pack_bf16(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
        }
        if (n >= WIDE) {
          put_block<WIDE>(block + (int64_t)row0 * ld + t.n0 + at, ld, w, p.rows - row0, turn);
        } else if (live) {
          put_some(block + row * ld + t.n0 + at, w, n);
        }
        __syncwarp();
      }
    } else {
#pragma unroll(mode_f32(MODE) ? 2 : 1)
      for (int c = 0; c < BN / 64; ++c) {
        const int at = half * (BN / 2) + 32 * c, n = p.cols - (t.n0 + at);
        uint32_t r[32];
        if (!empty) {
          tc_load32(r, acc + at);
          tc_landed(r);
        }
        if (n > 0 && !(empty && p.accumulate)) {
          float v[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = empty ? 0.0f : __uint_as_float(r[j]);
          if constexpr (mode_f32(MODE)) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += before[c][j];
          }
          put_piece<typename std::conditional<mode_f32(MODE), float, __nv_bfloat16>::type, MODE>(
              p, t, row, at, v, n, turn);
        }
        __syncwarp();   // the loads are the whole warp's
      }
    }
  }
}

// The ring of stages and the two accumulators as a role goes through them.
struct RingState {
  int s = 0, laps = 0;   // stage, and how often the ring has been gone through
  int n = 0;             // accumulators used
};

// Warp 8's lane: operand tiles into the ring.
template <int KIND, int CG, int BN>
__device__ __forceinline__ bool fill_tile(const TileArgs<KIND>& p, int i, RingState& r,
                                          TileShared<CG, BN>& sh, unsigned char* ring, unsigned rank) {
  const Tile t = tile_at<KIND, CG, BN>(p, i);
  for (int kt = 0; kt < t.nkt; ++kt) {
    if (!bar_wait<CG>(&sh.empty[r.s], (r.laps & 1) ^ 1, &sh.abort)) return false;
    unsigned char* a = ring + r.s * tile_stage_bytes(CG, BN);
    const uint32_t bar = CG == 1 ? st_smem(&sh.full[r.s]) : peer_smem(&sh.full[r.s], 0);
    if (rank == 0) bar_arrive_tx(&sh.full[r.s], CG * tile_stage_bytes(CG, BN));
    load_step<KIND, CG, BN>(p, t, kt, rank, a, a + kTileM * kTileK * 2, bar);
    if (++r.s == tile_stages(CG, BN)) r.s = 0, ++r.laps;
  }
  return true;
}

// Warp 9's lane (of a pair's first CTA): the products of a tile.
template <int KIND, int CG, int BN>
__device__ __forceinline__ bool multiply_tile(const TileArgs<KIND>& p, int i, RingState& r,
                                              TileShared<CG, BN>& sh, unsigned char* ring) {
  constexpr bool A_ACROSS = KIND == kWeight, B_ACROSS = KIND != kGate;
  constexpr uint32_t desc = product_desc(kTileM * CG, BN, A_ACROSS, B_ACROSS);
  constexpr uint32_t chunk = 64 * kTileK * 2;
  // 16 of the sum: 32 bytes along a swizzled row, or 16 rows of 128 bytes
  constexpr uint32_t a_step = A_ACROSS ? 2048 : 32, b_step = B_ACROSS ? 2048 : 32;
  const Tile t = tile_at<KIND, CG, BN>(p, i);
  if (t.nkt == 0) return true;
  for (int k0 = 0; k0 < t.nkt; k0 += t.span) {
    const int acc = r.n & 1, end = t.nkt - k0 < t.span ? t.nkt : k0 + t.span;
    if (!bar_wait<CG>(&sh.tempty[acc], ((r.n >> 1) & 1) ^ 1, &sh.abort)) return false;
    tc_fence_after();
    const uint32_t d = sh.tmem + acc * BN;
    for (int kt = k0; kt < end; ++kt) {
      if (!bar_wait<CG>(&sh.full[r.s], r.laps & 1, &sh.abort)) return false;
      tc_fence_after();
      const uint32_t a = st_smem(ring + r.s * tile_stage_bytes(CG, BN)), b = a + kTileM * kTileK * 2;
#pragma unroll
      for (int k = 0; k < kTileK / 16; ++k)
        tile_product<CG>(d, operand_desc(a + k * a_step, chunk), operand_desc(b + k * b_step, chunk),
                         desc, kt > k0 || k > 0);
      products_arrive<CG>(&sh.empty[r.s]);
      if (++r.s == tile_stages(CG, BN)) r.s = 0, ++r.laps;
    }
    products_arrive<CG>(&sh.tfull[acc]);
    ++r.n;
  }
  return true;
}

// What a tile's results are added to, towards the L2: this warp's rows, ahead of the
// tile before it, whose writing covers the way from memory.  16 languages of 40 rows,
// 6178 x 544: bf16 80 us without, 67 to 72 so, fp32 107 and 97; fp32 6178 x 534, not
// aligned, 158 and 142.  Not in kernels that need not add, whose registers it costs: fp32
// with nothing to add to 59 us without it, 62 with it; nor for turned bf16, where adding
// gains little or nothing (6178 x 534 121 us without, 117 with it; 533 wide 111, 121;
// 6716 x 6034 402, 407) and 533 wide with nothing to add to takes 81 us instead of 71.
template <int BN, int CG>
__device__ __forceinline__ void fetch_tile(const TileArgs<kWeight>& p, int i, unsigned rank) {
  if (i >= p.tiles) return;
  const Tile t = tile_at<kWeight, CG, BN>(p, i);
  const int wid = threadIdx.x >> 5;
  const int row = t.m0 + (int)rank * kTileM + (wid & 3) * 32 + (threadIdx.x & 31);
  const int col = t.n0 + (wid >> 2) * (BN / 2), elem = p.out_dtype == BKMOO_F32 ? 4 : 2;
  const int bytes = (p.cols - col < BN / 2 ? p.cols - col : BN / 2) * elem;
  if (t.nkt == 0 || row >= p.rows || bytes <= 0) return;
  const char* q = static_cast<const char*>(p.out[t.g]) + ((int64_t)row * p.cols + col) * elem;
  for (int b = 0; b < bytes; b += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + b));
  asm volatile("prefetch.global.L2 [%0];" ::"l"(q + bytes - 1));
}

// Warps 0 to 7: a finished tile to memory.
template <int KIND, int CG, int BN, int MODE>
__device__ __forceinline__ bool drain_tile(const TileArgs<KIND>& p, int i, RingState& r,
                                           TileShared<CG, BN>& sh, float* turn, unsigned rank) {
  const int wid = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = wid & 3, half = wid >> 2;
  const Tile t = tile_at<KIND, CG, BN>(p, i);
  const int row = t.m0 + (int)rank * kTileM + quarter * 32 + lane;
  const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
  auto wait = [&]() {
    const bool ok = bar_wait<CG>(&sh.tfull[r.n & 1], (r.n >> 1) & 1, &sh.abort);
    if (!__all_sync(0xffffffffu, ok)) return false;
    tc_fence_after();
    return true;
  };
  auto release = [&]() {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) {
      if (rank == 0) bar_arrive(&sh.tempty[r.n & 1]);
      else bar_arrive_at(peer_smem(&sh.tempty[r.n & 1], 0));
    }
    ++r.n;
  };
  if constexpr (KIND == kWeight && mode_f32(MODE)) {
    float sum[BN / 64][32];          // of the pieces but the last
#pragma unroll
    for (int c = 0; c < BN / 64; ++c)
#pragma unroll
      for (int j = 0; j < 32; ++j) sum[c][j] = 0.0f;
#pragma unroll 1
    for (int k0 = 0; k0 + t.span < t.nkt; k0 += t.span) {
      if (!wait()) return false;
#pragma unroll
      for (int c = 0; c < BN / 64; ++c) {
        uint32_t v[32];
        tc_load32(v, sh.tmem + lanes + (r.n & 1) * BN + half * (BN / 2) + 32 * c);
        tc_landed(v);
#pragma unroll
        for (int j = 0; j < 32; ++j) sum[c][j] += __uint_as_float(v[j]);
      }
      release();
    }
    if (t.nkt > 0 && !wait()) return false;
    take_tile<KIND, BN, MODE>(p, t, row, half, sh.tmem + lanes + (r.n & 1) * BN, t.nkt == 0,
                              turn + wid * (kTurnBytes / 4), sum);
  } else {
    if (t.nkt > 0 && !wait()) return false;
    take_tile<KIND, BN, MODE>(p, t, row, half, sh.tmem + lanes + (r.n & 1) * BN, t.nkt == 0,
                              turn + wid * (kTurnBytes / 4), nullptr);
  }
  if (t.nkt > 0) release();
  return true;
}

template <int KIND, int CG, int BN, int MODE>
__global__ void __launch_bounds__(kTileThreads, 1)
    tile_gemm_kernel(const __grid_constant__ TileArgs<KIND> p) {
  constexpr int S = tile_stages(CG, BN);
  extern __shared__ unsigned char raw[];
  __shared__ TileShared<CG, BN> sh;
  unsigned char* ring = raw + ((1024 - (st_smem(raw) & 1023)) & 1023);
  float* turn = reinterpret_cast<float*>(ring + S * tile_stage_bytes(CG, BN));
  const int wid = threadIdx.x >> 5;
  const unsigned rank = CG == 1 ? 0 : cluster_rank();

  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      bar_init(&sh.full[i], 1);
      bar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(&sh.tfull[i], 1);
      bar_init(&sh.tempty[i], CG * kTileEpilogueWarps);
    }
    bar_init(&sh.drain, 1);
    sh.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (wid == kTileEpilogueWarps + 1) {
    tmem_alloc<CG>(&sh.tmem, 2 * BN);
    tc_fence_before();
  }
  __syncthreads();
  if (CG == 2) cluster_sync();
  tc_fence_after();
  grid_wait();
  const uint32_t tmem = sh.tmem;

  // f over this CTA's tiles, until it gives up (a whole warp as one, or one lane), and
  // `ahead` over kWeight's, each before the f of the tile before it
  auto each = [&](auto f, auto ahead) {
    int i;
    bool on = true;
    if constexpr (KIND == kBoth) {
      Walk walk(blockIdx.x / CG, gridDim.x / CG, p.in.tiles, p.w.tiles, p.head_start);
      int set = walk.next(i);
      if (set == 2) ahead(p.w, i);
      while (on && set != 0) {
        int j;
        const int then = walk.next(j);
        if (then == 2) ahead(p.w, j);
        if (set == 1) on = f(std::integral_constant<int, kInput>(), p.in, i);
        else on = f(std::integral_constant<int, kWeight>(), p.w, i);
        set = then;
        i = j;
      }
    } else {
      i = blockIdx.x / CG;
      ahead(p, i);
      for (; on && i < p.tiles; i += gridDim.x / CG) {
        ahead(p, i + gridDim.x / CG);
        on = f(std::integral_constant<int, KIND>(), p, i);
      }
    }
  };
  auto none = [](const auto&, int) {};
  RingState r;
  bool feed = true;
  if constexpr (KIND == kGate) feed = !p.withhold;
  if (wid == kTileEpilogueWarps) {
    if (feed && elect_one()) {
      each([&](auto kind, const auto& q, int i) {
        return fill_tile<decltype(kind)::value, CG, BN>(q, i, r, sh, ring, rank);
      }, none);
      // every copy has landed and been used before the CTA ends
      for (int i = 0; i < S; ++i) {
        if (!bar_wait<CG>(&sh.empty[r.s], (r.laps & 1) ^ 1, &sh.abort) && rank == 0 && r.laps > 0) {
          int no = 0;
          bar_wait<CG>(&sh.full[r.s], (r.laps & 1) ^ 1, &no);
        }
        if (++r.s == S) r.s = 0, ++r.laps;
      }
    }
  } else if (wid == kTileEpilogueWarps + 1) {
    if (rank == 0 && elect_one()) {
      each([&](auto kind, const auto& q, int i) {
        return multiply_tile<decltype(kind)::value, CG, BN>(q, i, r, sh, ring);
      }, none);
      if (sh.abort) {
        // no product is in flight when tensor memory is handed back
        int no = 0;
        products_arrive<CG>(&sh.drain);
        bar_wait<CG>(&sh.drain, 0, &no);
      }
    }
  } else {
    each([&](auto kind, const auto& q, int i) {
      return drain_tile<decltype(kind)::value, CG, BN, MODE>(q, i, r, sh, turn, rank);
    }, [&](const auto& q, int i) {
      if constexpr (mode_ahead(MODE)) fetch_tile<BN, CG>(q, i, rank);
      __syncwarp();
    });
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();
  tc_fence_after();
  if (wid == kTileEpilogueWarps + 1) tmem_free<CG>(tmem, 2 * BN);
  if (threadIdx.x == 0 && sh.abort) report_give_up(p.status);
}

// The kernels, one translation unit each (nvcc runs them side by side).
const void* tile_gate_fn(int cg, int bn);
const void* tile_weight_fn(int cg, int bn, int mode);
const void* tile_both_fn(int cg, int bn, int mode);

}  // namespace bkmoo
