// Queries and keys normed head by head, times a weight, and rotated by their position, and
// the backward pass with the weights' gradients apart by language (include/bkmoo.h).
//
// r = 1 / sqrt(mean(x^2) + eps), n = x r, y = w n, and pairs (a, b) of y turned by
// pos f_i: a cos - b sin, b cos + a sin.  Back: dy is do turned the other way,
// dw = sum dy n, dx = r (w dy - n mean(w dy n)).  Everything of a head is in the registers
// of 1 to 16 lanes, 16 elements each, the two halves of 8 pairs: one pass, bound by memory.
//
// A position's angle in turns is pos f / 2 pi, of which only the fraction counts.  The
// frequency is kept as a 64-bit fraction of a turn, so that the product modulo 2^64 is that
// fraction, without floating point in 64 bits.  The product is exact; the angle is off by what
// the frequency is, times the position: f / 2 pi has two roundings in 64-bit floating point (2^-52 of
// itself) and is cut to 2^-64 of a turn; and by 2^-26 of a turn where the fraction becomes fp32.
#include <math.h>

#include "tile_host.cuh"
#include "row_ops.cuh"

namespace bkmoo {
namespace {

constexpr int kQkThreads = 128;
constexpr int kQkWarps = kQkThreads / 32;
constexpr int kMaxHead = 256;
constexpr int kForwardCtas = 5, kBackwardCtas = 4;     // on an SM
constexpr int kAhead = 3;               // steps of a warp whose loads are on their way

struct QkSide {
  const __nv_bfloat16 *x, *dout;
  __nv_bfloat16* out;                   // forward: the result; backward: dx
  const void* w;
  int64_t ld, ld_dout, ld_out;          // from token to token
  int32_t heads, steps;                 // steps: groups of heads that a warp takes at once
};
struct QkArgs {
  QkSide side[2];
  const void* pos;
  int32_t id_bytes, w_f32;
  int32_t hd, rot;
  float eps, inv_hd;
  int64_t T;
  uint64_t turn[kMaxHead / 2];          // 2^64 f / 2 pi
};

// 16 numbers of each of a head's lanes, four by four, those of neighbouring lanes side by side:
// eight lanes read 128 bytes in a row.
struct Numbers {
  float4 v[4][16];
  __device__ __forceinline__ float& at(int l, int j) { return reinterpret_cast<float*>(&v[j >> 2][l])[j & 3]; }
  __device__ __forceinline__ void get(int l, float (&x)[16]) const {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 f = v[q][l];
      x[4 * q] = f.x, x[4 * q + 1] = f.y, x[4 * q + 2] = f.z, x[4 * q + 3] = f.w;
    }
  }
};
// The cos and sin of a token's pairs, 8 a lane, by a warp.
template <bool NEIGHBOURS>
__device__ __forceinline__ void angles(const QkArgs& a, uint64_t pos, int lane, Numbers& room) {
  __syncwarp();
  for (int i = lane; i < a.rot / 2; i += 32) {
    // half turns in [-1, 1)
    const float half = __int2float_rn((int32_t)((pos * a.turn[i] + 0x80000000ull) >> 32)) * 0x1p-31f;
    // where the lane that has the pair keeps it (Place)
    const bool second = NEIGHBOURS && i >= a.hd / 4;
    const int k = second ? i - a.hd / 4 : i, l = NEIGHBOURS ? k >> 2 : k >> 3, j = NEIGHBOURS ? (second ? 4 : 0) + (k & 3) : k & 7;
    sincospif(half, &room.at(l, 8 + j), &room.at(l, j));
  }
  __syncwarp();
}
// None is turned, at first.
__device__ __forceinline__ void no_angles(int lane, Numbers& room) {
  for (int i = lane; i < 128; i += 32) room.at(i >> 3, i & 7) = 1.0f, room.at(i >> 3, 8 + (i & 7)) = 0.0f;
}

// Where a lane's 16 elements of a head lie: two vectors of 8, whose pairs are between them or within
// each.  Neighbouring lanes' vectors are neighbours: a line of memory is asked for once.
struct Place {
  int lo, hi;                           // columns
  bool live;
};
template <bool NEIGHBOURS>
__device__ __forceinline__ Place place_of_lane(const QkArgs& a, int l) {
  Place p;
  p.live = 16 * l < a.hd;
  if (NEIGHBOURS) {
    p.lo = 8 * l;
    p.hi = p.lo + a.hd / 2;
  } else if (16 * l < a.rot) {
    p.lo = 8 * l;
    p.hi = p.lo + a.rot / 2;
  } else {
    p.lo = a.rot / 2 + 8 * l;
    p.hi = p.lo + (a.hd - a.rot) / 2;
  }
  return p;
}
// y: the lane's elements, the vector at lo and then the one at hi, turned back by g, 8 cos and
// 8 sin.
template <bool NEIGHBOURS>
__device__ __forceinline__ void turn_back(float (&y)[16], const float (&g)[16]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float& a = y[NEIGHBOURS ? 2 * j : j];
    float& b = y[NEIGHBOURS ? 2 * j + 1 : j + 8];
    const float x = a;
    a = fmaf(b, g[j + 8], x * g[j]);
    b = fmaf(-x, g[j + 8], b * g[j]);
  }
}
__device__ __forceinline__ float weight_at(const QkArgs& a, const void* w, int c) {
  return a.w_f32 ? static_cast<const float*>(w)[c] : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[c]);
}
template <bool NEIGHBOURS>
__device__ __forceinline__ void get_weights(const QkArgs& a, const void* w, Numbers& to) {
  for (int i = threadIdx.x; i < 256; i += kQkThreads) {
    const int l = i >> 4, j = i & 15;
    const Place p = place_of_lane<NEIGHBOURS>(a, l);
    to.at(l, j) = p.live ? weight_at(a, w, (j < 8 ? p.lo : p.hi) + (j & 7)) : 0.0f;
  }
}
// Loads go to shared memory, each lane's to a place of its own that only it reads: a copy
// that is on its way holds no register.
struct Pair {
  uint4 lo[32], hi[32];
};
// (Where !live nothing is read and the place becomes 0.)
__device__ __forceinline__ void copy16(uint4* to, const __nv_bfloat16* from, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from),
               "r"(live ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void copy_pair(Pair& to, const __nv_bfloat16* head, const __nv_bfloat16* any, const Place& p, int lane,
                                          bool live) {
  copy16(&to.lo[lane], live ? head + p.lo : any, live);
  copy16(&to.hi[lane], live ? head + p.hi : any, live);
}
__device__ __forceinline__ int next_slot(int slot) { return slot == kAhead - 1 ? 0 : slot + 1; }
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// All but the newest kAhead - 1 steps' copies have come.
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory"); }
__device__ __forceinline__ void get_pair(const Pair& v, int lane, float (&x)[16]) {
  float a[8], b[8];
  unpack(v.lo[lane], a);
  unpack(v.hi[lane], b);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = a[j], x[j + 8] = b[j];
}
__device__ __forceinline__ void store_pair(__nv_bfloat16* head, const Place& p, const float (&x)[16]) {
  const float a[8] = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]},
              b[8] = {x[8], x[9], x[10], x[11], x[12], x[13], x[14], x[15]};
  *reinterpret_cast<uint4*>(head + p.lo) = repack(a);
  *reinterpret_cast<uint4*>(head + p.hi) = repack(b);
}
template <int G>
__device__ __forceinline__ float over_head(float v) {
#pragma unroll
  for (int w = G / 2; w > 0; w >>= 1) v += __shfl_xor_sync(0xffffffffu, v, w);
  return v;
}

// A warp's way through steps: 32 / G heads of a token, its queries' and then its keys', token after
// token.  at: the lane's head in one array; over: the heads from there on, 0 or less behind the last.
template <class E>
struct Way {
  int64_t t;
  int step, over;
  E* at;
};

// G lanes a head.  A warp takes a run of steps.  Bound by memory: 8192 tokens of 32 + 8 heads of
// 128 take 30 us (5.6 TB/s), and 29 in a copy of this kernel that copies and computes nothing.
// 5 CTAs on an SM and 3 steps ahead: 6 and 7 CTAs 30.3 and 31.9, 6 steps 30.5.
template <int G, bool NEIGHBOURS>
__global__ void __launch_bounds__(kQkThreads, kForwardCtas) qk_norm_kernel(const __grid_constant__ QkArgs a, const int64_t each) {
  grid_wait();
  grid_release();
  __shared__ Numbers room[kQkWarps], weights[2];
  __shared__ Pair ring[kQkWarps][kAhead];
  constexpr int kHeads = 32 / G;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int queries = a.side[0].heads, heads = queries + a.side[1].heads, per = (heads + kHeads - 1) / kHeads;
  // the first steps with a key and without a query
  const int some = queries / kHeads, none = (queries + kHeads - 1) / kHeads, step_elems = kHeads * a.hd;
  const int64_t total = a.T * per, from = ((int64_t)blockIdx.x * kQkWarps + wid) * each;
  const int64_t to = from + each < total ? from + each : total;
  const int steps = from < to ? (int)(to - from) : 0;
  const Place p = place_of_lane<NEIGHBOURS>(a, lane % G);
  auto side_of = [&](int step) { return step * kHeads + lane / G >= queries; };
  auto set = [&](auto& w, auto* const x, int64_t ld) {       // to its token's and step's head
    const int head = w.step * kHeads + lane / G;
    w.over = p.live ? heads - head : 0;
    w.at = x + w.t * ld + (int64_t)(head >= queries ? head - queries : head) * a.hd;
  };
  auto set_in = [&](Way<const __nv_bfloat16>& w) { set(w, a.side[side_of(w.step)].x, a.side[side_of(w.step)].ld); };
  auto set_out = [&](Way<__nv_bfloat16>& w) { set(w, a.side[side_of(w.step)].out, a.side[side_of(w.step)].ld_out); };
  Way<const __nv_bfloat16> there;
  Way<__nv_bfloat16> here;
  here.t = there.t = from / per;
  here.step = there.step = (int)(from % per);
  set_in(there);
  set_out(here);
  // whether a token begins, or its keys
  auto next = [&](auto& w) {
    w.over -= kHeads;
    w.at += step_elems;
    if (++w.step < per) return w.step == some || w.step == none;
    w.step = 0;
    ++w.t;
    return true;
  };
  int ahead = 0, slot = 0, slot_there = 0;
  auto fetch = [&]() {
    const bool live = there.over > 0 && ahead < steps;
    copy_pair(ring[wid][slot_there], there.at, a.side[0].x, p, lane, live);
    copies_end();
    slot_there = next_slot(slot_there);
    if (next(there)) set_in(there);
    ++ahead;
  };
#pragma unroll
  for (int j = 0; j < kAhead - 1; ++j) fetch();
  for (int k = 0; k < 2; ++k) get_weights<NEIGHBOURS>(a, a.side[k].w, weights[k]);
  no_angles(lane, room[wid]);
  __syncthreads();
  int64_t pos = steps > 0 ? load_id(a.pos, a.id_bytes, here.t) : 0;
  bool begins = true, new_token = true;
  // r times these of the pair's two elements: the rotation of the weighed ones
  float ca[8], sa[8], cb[8], sb[8];
  for (int i = 0; i < steps; ++i) {
    fetch();
    if (begins) {
      if (new_token) {
        angles<NEIGHBOURS>(a, (uint64_t)pos, lane, room[wid]);
        if (here.t + 1 < a.T) pos = load_id(a.pos, a.id_bytes, here.t + 1);
      }
      float g[16], w[16];
      room[wid].get(lane % G, g);
      weights[side_of(here.step)].get(lane % G, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float wa = w[NEIGHBOURS ? 2 * j : j], wb = w[NEIGHBOURS ? 2 * j + 1 : j + 8];
        ca[j] = wa * g[j];
        sa[j] = wa * g[j + 8];
        cb[j] = wb * g[j];
        sb[j] = wb * g[j + 8];
      }
    }
    copies_wait();
    float x[16], sum = 0.0f;
    get_pair(ring[wid][slot], lane, x);
    slot = next_slot(slot);
#pragma unroll
    for (int j = 0; j < 16; ++j) sum = fmaf(x[j], x[j], sum);
    const float r = rsqrtf(fmaf(over_head<G>(sum), a.inv_hd, a.eps));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float& u = x[NEIGHBOURS ? 2 * j : j];
      float& v = x[NEIGHBOURS ? 2 * j + 1 : j + 8];
      const float y = fmaf(-v, sb[j], u * ca[j]);
      v = r * fmaf(u, sa[j], v * cb[j]);
      u = r * y;
    }
    if (here.over > 0) store_pair(here.at, p, x);
    const int64_t t = here.t;
    begins = next(here);
    if (begins) set_out(here);
    new_token = here.t != t;
  }
  copies_wait_all();
}

// The backward pass by CTAs that each take a run of one side's and one language's steps, and leave
// their sums of the weights' gradients.  8192 tokens of 32 + 8 heads of 128 in 4 languages take
// 44 us (5.8 TB/s), of which 3 are the sums' kernel.  4 CTAs on an SM: when it took 46, 5 CTAs, whose
// registers go to memory, took 53, 3 CTAs 55, and tokens dealt out in turn instead of in runs 53.
// w and the angles are read from shared memory for every step: the registers hold the sums.
struct QkRuns {
  int32_t K, weights;
  int32_t first[2 * kMaxK + 1];         // CTAs of (side, language), side by side
  int64_t rows[kMaxK + 1];
  float* part;                          // [CTA][hd]
};
template <int G, bool NEIGHBOURS>
__global__ void __launch_bounds__(kQkThreads, kBackwardCtas) qk_norm_grad_kernel(const __grid_constant__ QkArgs a,
                                                                  const __grid_constant__ QkRuns q) {
  grid_wait();
  grid_release();
  __shared__ Numbers room[kQkWarps], weights;
  __shared__ Pair ring[kQkWarps][kAhead][2];             // x, dout
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, l = lane % G;
  int run = 0;
  while ((int)blockIdx.x >= q.first[run + 1]) ++run;
  const int k = run / q.K, lang = run % q.K, ctas = q.first[run + 1] - q.first[run];
  const QkSide& s = a.side[k];
  const int64_t all = (q.rows[lang + 1] - q.rows[lang]) * s.steps, warps = (int64_t)ctas * kQkWarps;
  const int64_t me = (int64_t)(blockIdx.x - q.first[run]) * kQkWarps + wid;
  const int64_t each = (all + warps - 1) / warps;
  const int64_t from = me * each < all ? me * each : all, to = from + each < all ? from + each : all;
  const Place p = place_of_lane<NEIGHBOURS>(a, l);
  const int steps = (int)(to - from), step_elems = 32 / G * a.hd;
  // the lane's head in each array, and what leads from a token's last to the next one's first
  const int64_t t0 = q.rows[lang] + from / s.steps;
  const int step0 = (int)(from % s.steps), head0 = lane / G;
  const int64_t back = (int64_t)(s.steps - 1) * step_elems, in = (int64_t)(step0 * (32 / G) + head0) * a.hd;
  const __nv_bfloat16 *at_x = s.x + t0 * s.ld + in, *at_d = s.dout + t0 * s.ld_dout + in;
  __nv_bfloat16* at_out = s.out + t0 * s.ld_out + in;
  int step = step0, step_there = step0, ahead = 0, slot = 0, slot_there = 0;
  int64_t t = t0;
  auto live_at = [&](int step) { return p.live && step * (32 / G) + head0 < s.heads; };
  auto fetch = [&]() {
    Pair* r = ring[wid][slot_there];
    slot_there = next_slot(slot_there);
    const bool live = ahead < steps && live_at(step_there);
    copy_pair(r[0], at_x, s.x, p, lane, live);
    copy_pair(r[1], at_d, s.x, p, lane, live);
    copies_end();
    const bool end = ++step_there == s.steps;
    if (end) step_there = 0;
    at_x += end ? s.ld - back : step_elems;
    at_d += end ? s.ld_dout - back : step_elems;
    ++ahead;
  };
#pragma unroll
  for (int j = 0; j < kAhead - 1; ++j) fetch();
  get_weights<NEIGHBOURS>(a, s.w, weights);
  no_angles(lane, room[wid]);
  __syncthreads();
  float dw[16] = {};
  int64_t pos = steps > 0 ? load_id(a.pos, a.id_bytes, t) : 0;
  bool new_token = true;
  for (int i = 0; i < steps; ++i) {
    fetch();
    if (new_token) {
      angles<NEIGHBOURS>(a, (uint64_t)pos, lane, room[wid]);
      if (t + 1 < a.T) pos = load_id(a.pos, a.id_bytes, t + 1);
    }
    const bool live = live_at(step);
    copies_wait();
    const Pair* v = ring[wid][slot];
    slot = next_slot(slot);
    float x[16], d[16], w[16], sum = 0.0f, dot = 0.0f;
    get_pair(v[1], lane, d);
    room[wid].get(l, w);                // (w and the angles stay in shared memory: registers are short)
    turn_back<NEIGHBOURS>(d, w);
    get_pair(v[0], lane, x);
    weights.get(l, w);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      sum = fmaf(x[j], x[j], sum);
      w[j] *= d[j];
      dot = fmaf(w[j], x[j], dot);
    }
    // (0 beyond the last head: without eps, 1 / sqrt(0) would leave NaN in dw)
    const float squares = over_head<G>(sum), r = live ? rsqrtf(fmaf(squares, a.inv_hd, a.eps)) : 0.0f;
    const float c = over_head<G>(dot) * r * r * a.inv_hd;     // mean(w dy n) / n's x
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float n = x[j] * r;
      dw[j] = fmaf(d[j], n, dw[j]);
      d[j] = r * fmaf(-x[j], c, w[j]);
    }
    if (live) store_pair(at_out, p, d);
    new_token = ++step == s.steps;
    at_out += new_token ? s.ld_out - back : step_elems;
    if (new_token) step = 0, ++t;
  }
  copies_wait_all();
  if (!q.weights) return;
  __shared__ float sums[kQkWarps][kMaxHead];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
#pragma unroll
    for (int h = G; h < 32; h *= 2) dw[j] += __shfl_xor_sync(0xffffffffu, dw[j], h);
    if (lane < G && p.live) sums[wid][(j < 8 ? p.lo : p.hi) + (j & 7)] = dw[j];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.hd; c += kQkThreads) {
    float v = 0.0f;
    for (int i = 0; i < kQkWarps; ++i) v += sums[i][c];
    q.part[(int64_t)blockIdx.x * a.hd + c] = v;
  }
}

// The CTAs' sums of one side's and one language's columns joined in the order of the CTAs,
// 32 columns a CTA.
struct QkWeightGrads {
  void* dw[2 * kMaxK];
  int32_t first[2 * kMaxK + 1];
  const float* part;
  int32_t hd, f32, accumulate;
};
__global__ void __launch_bounds__(1024) qk_weight_kernel(const __grid_constant__ QkWeightGrads a) {
  grid_wait();
  grid_release();
  const int run = blockIdx.x, c = blockIdx.y * 32 + (threadIdx.x & 31), at = threadIdx.x >> 5;
  __shared__ float sums[32][32];
  float v = 0.0f;
  if (c < a.hd)
    for (int i = a.first[run] + at; i < a.first[run + 1]; i += 32) v += a.part[(int64_t)i * a.hd + c];
  sums[at][threadIdx.x & 31] = v;
  __syncthreads();
  if (at != 0 || c >= a.hd) return;
  for (int i = 1; i < 32; ++i) v += sums[i][threadIdx.x];
  if (a.f32) {
    float* p = static_cast<float*>(a.dw[run]) + c;
    *p = a.accumulate ? *p + v : v;
  } else {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(a.dw[run]) + c;
    *p = __float2bfloat16_rn(a.accumulate ? __bfloat162float(*p) + v : v);
  }
}

template <int G>
const void* forward_fn(bool n) {
  return n ? (const void*)qk_norm_kernel<G, true> : (const void*)qk_norm_kernel<G, false>;
}
template <int G>
const void* backward_fn(bool n) {
  return n ? (const void*)qk_norm_grad_kernel<G, true> : (const void*)qk_norm_grad_kernel<G, false>;
}

int lanes_of(int64_t hd) {
  int g = 1;
  while (16 * g < hd) g *= 2;
  return g;
}

bool heads_ok(const void* p, int64_t T, int64_t heads, int64_t hd, int64_t ld) {
  return T == 0 || (aligned_at(p, 16) && ld >= heads * hd && ld % 8 == 0 && ld <= ((int64_t)1 << 38));
}
bool qk_sizes_ok(int64_t T, int64_t hq, int64_t hk, int64_t hd, const double* freq, int64_t rot, double eps) {
  if (T < 0 || T > ((int64_t)1 << 31) - 1024 || hq < 1 || hk < 1 || hq > 65536 || hk > 65536 || hd < 16 ||
      hd > kMaxHead || hd % 16 || rot < 0 || rot > hd || rot % 16 || !(eps >= 0.0) || !std::isfinite(eps) ||
      (rot > 0 && !freq))
    return false;
  for (int64_t i = 0; i < rot / 2; ++i)
    if (!std::isfinite(freq[i])) return false;
  return true;
}
void fill(QkArgs& a, int64_t T, int64_t hq, int64_t hk, int64_t hd, const double* freq, int64_t rot, double eps) {
  const int at_once = 32 / lanes_of(hd);
  a.side[0].heads = (int32_t)hq;
  a.side[1].heads = (int32_t)hk;
  for (int i = 0; i < 2; ++i) a.side[i].steps = (a.side[i].heads + at_once - 1) / at_once;
  a.hd = (int32_t)hd;
  a.rot = (int32_t)rot;
  a.eps = (float)eps;
  a.inv_hd = 1.0f / (float)hd;
  a.T = T;
  for (int64_t i = 0; i < rot / 2; ++i) {
    const double turns = freq[i] * 0.15915494309189533577;        // 1 / 2 pi
    const double part = (turns - std::floor(turns)) * 18446744073709551616.0;     // exact
    a.turn[i] = part < 18446744073709551616.0 ? (uint64_t)part : 0;
  }
}
constexpr int kMostCtas = 2048;         // of the backward pass, whose sums the workspace holds

bool places_ok(void* const* dw, int32_t K, int32_t dtype) {
  for (int k = 0; k < K; ++k)
    if (!aligned_at(dw[k], float_bytes(dtype))) return false;
  return true;
}

}  // namespace
}  // namespace bkmoo

using namespace bkmoo;

extern "C" int bkmoo_qk_norm_forward(const void* q, int64_t ldq, const void* k, int64_t ldk,
                                     const void* w_q, const void* w_k, int32_t w_dtype, int64_t T,
                                     int64_t q_heads, int64_t k_heads, int64_t head_dim,
                                     const void* positions, int32_t id_bytes, const double* inv_freq,
                                     int64_t rot, int32_t interleaved, double eps, void* q_out,
                                     int64_t ldq_out, void* k_out, int64_t ldk_out, void* stream) {
  if (!is_float(w_dtype) || !is_id(id_bytes) || !qk_sizes_ok(T, q_heads, k_heads, head_dim, inv_freq, rot, eps) ||
      !aligned_at(w_q, float_bytes(w_dtype)) || !aligned_at(w_k, float_bytes(w_dtype)))
    return BKMOO_ERR_INVALID;
  if (T == 0) return BKMOO_OK;
  if (!heads_ok(q, T, q_heads, head_dim, ldq) || !heads_ok(k, T, k_heads, head_dim, ldk) ||
      !heads_ok(q_out, T, q_heads, head_dim, ldq_out) || !heads_ok(k_out, T, k_heads, head_dim, ldk_out) ||
      (q == q_out && ldq != ldq_out) || (k == k_out && ldk != ldk_out) || !aligned_at(positions, id_bytes))
    return BKMOO_ERR_INVALID;
  QkArgs a = {};
  fill(a, T, q_heads, k_heads, head_dim, inv_freq, rot, eps);
  a.side[0].x = static_cast<const __nv_bfloat16*>(q);
  a.side[1].x = static_cast<const __nv_bfloat16*>(k);
  a.side[0].out = static_cast<__nv_bfloat16*>(q_out);
  a.side[1].out = static_cast<__nv_bfloat16*>(k_out);
  a.side[0].w = w_q;
  a.side[1].w = w_k;
  a.side[0].ld = ldq;
  a.side[1].ld = ldk;
  a.side[0].ld_out = ldq_out;
  a.side[1].ld_out = ldk_out;
  a.pos = positions;
  a.id_bytes = id_bytes;
  a.w_f32 = w_dtype == BKMOO_F32;
  const int g = lanes_of(head_dim);
  const void* fn = g == 1   ? forward_fn<1>(interleaved)
                   : g == 2 ? forward_fn<2>(interleaved)
                   : g == 4 ? forward_fn<4>(interleaved)
                   : g == 8 ? forward_fn<8>(interleaved)
                            : forward_fn<16>(interleaved);
  int ctas = 0;
  if (tile_sms(&ctas) != BKMOO_OK) return BKMOO_ERR_CUDA;
  ctas *= kForwardCtas;
  const int at_once = 32 / g;
  const int64_t total = T * ((q_heads + k_heads + at_once - 1) / at_once);
  int64_t each = (total + (int64_t)ctas * kQkWarps - 1) / ((int64_t)ctas * kQkWarps);
  const int64_t grid = (total + each * kQkWarps - 1) / (each * kQkWarps);
  void* list[] = {&a, &each};
  return launch_behind(fn, dim3((unsigned)grid), dim3(kQkThreads), list, 0, static_cast<cudaStream_t>(stream),
                       true) == cudaSuccess
             ? BKMOO_OK
             : BKMOO_ERR_CUDA;
}

extern "C" int bkmoo_qk_norm_backward_workspace_size(int64_t head_dim, size_t* bytes) {
  if (!bytes || head_dim < 16 || head_dim > kMaxHead || head_dim % 16) return BKMOO_ERR_INVALID;
  *bytes = (size_t)kMostCtas * (size_t)head_dim * sizeof(float);
  return BKMOO_OK;
}

extern "C" int bkmoo_qk_norm_backward(const void* dq_out, int64_t ld_dq_out, const void* dk_out,
                                      int64_t ld_dk_out, const void* q, int64_t ldq, const void* k,
                                      int64_t ldk, const void* w_q, const void* w_k, int32_t w_dtype,
                                      int64_t T, int64_t q_heads, int64_t k_heads, int64_t head_dim,
                                      const void* positions, int32_t id_bytes, const double* inv_freq,
                                      int64_t rot, int32_t interleaved, double eps, int32_t K,
                                      const int64_t* rows, void* dq, int64_t ld_dq, void* dk,
                                      int64_t ld_dk, void* const* dw_q, void* const* dw_k,
                                      int32_t dw_dtype, int32_t accumulate, void* ws, size_t ws_bytes,
                                      void* stream) {
  const bool weights = dw_q || dw_k;
  if (!is_float(w_dtype) || !is_id(id_bytes) || !is_float(dw_dtype) ||
      !qk_sizes_ok(T, q_heads, k_heads, head_dim, inv_freq, rot, eps) || !languages_ok(rows, K, T) ||
      !aligned_at(w_q, float_bytes(w_dtype)) || !aligned_at(w_k, float_bytes(w_dtype)) ||
      (weights && (!dw_q || !dw_k || !places_ok(dw_q, K, dw_dtype) || !places_ok(dw_k, K, dw_dtype))) ||
      (weights && !aligned_at(ws, 256)) || !heads_ok(q, T, q_heads, head_dim, ldq) ||
      !heads_ok(k, T, k_heads, head_dim, ldk) || !heads_ok(dq_out, T, q_heads, head_dim, ld_dq_out) ||
      !heads_ok(dk_out, T, k_heads, head_dim, ld_dk_out) || !heads_ok(dq, T, q_heads, head_dim, ld_dq) ||
      !heads_ok(dk, T, k_heads, head_dim, ld_dk) ||
      (T > 0 && ((dq == dq_out && ld_dq != ld_dq_out) || (dk == dk_out && ld_dk != ld_dk_out) ||
                 !aligned_at(positions, id_bytes))))
    return BKMOO_ERR_INVALID;
  if (weights) {
    const void* all[2 * kMaxK];
    for (int l = 0; l < K; ++l) all[l] = dw_q[l], all[K + l] = dw_k[l];
    if (!apart(all, 2 * K, (size_t)head_dim * float_bytes(dw_dtype))) return BKMOO_ERR_INVALID;
  }
  size_t need = 0;
  if (bkmoo_qk_norm_backward_workspace_size(head_dim, &need) != BKMOO_OK) return BKMOO_ERR_INVALID;
  if (weights && ws_bytes < need) return BKMOO_ERR_WORKSPACE;
  if (T == 0 && (!weights || accumulate)) return BKMOO_OK;
  QkArgs a = {};
  fill(a, T, q_heads, k_heads, head_dim, inv_freq, rot, eps);
  const void* x[2] = {q, k};
  const void* d[2] = {dq_out, dk_out};
  void* out[2] = {dq, dk};
  const void* w[2] = {w_q, w_k};
  const int64_t ld[2] = {ldq, ldk}, ld_dout[2] = {ld_dq_out, ld_dk_out}, ld_out[2] = {ld_dq, ld_dk};
  for (int i = 0; i < 2; ++i) {
    QkSide& s = a.side[i];
    s.x = static_cast<const __nv_bfloat16*>(x[i]);
    s.dout = static_cast<const __nv_bfloat16*>(d[i]);
    s.out = static_cast<__nv_bfloat16*>(out[i]);
    s.w = w[i];
    s.ld = ld[i];
    s.ld_dout = ld_dout[i];
    s.ld_out = ld_out[i];
  }
  a.pos = positions;
  a.id_bytes = id_bytes;
  a.w_f32 = w_dtype == BKMOO_F32;
  const int g = lanes_of(head_dim);
  const void* fn = g == 1   ? backward_fn<1>(interleaved)
                   : g == 2 ? backward_fn<2>(interleaved)
                   : g == 4 ? backward_fn<4>(interleaved)
                   : g == 8 ? backward_fn<8>(interleaved)
                            : backward_fn<16>(interleaved);
  int ctas = 0;
  if (tile_sms(&ctas) != BKMOO_OK) return BKMOO_ERR_CUDA;
  ctas *= kBackwardCtas;
  // A side's and a language's last CTA is not full.  With those all are to be on the card at
  // once: the few that were not would begin when the others end.
  if (ctas > kMostCtas) ctas = kMostCtas;
  ctas -= 2 * K;
  if (ctas < 1) ctas = 1;
  QkRuns r = {};
  r.K = K;
  r.weights = weights;
  r.part = static_cast<float*>(ws);
  // A token costs its steps and its angles, of which 256 are about as long as a step: 8680 tokens of
  // 16 + 2 heads of 256 took 81 us with CTAs dealt out by steps alone.
  int64_t cost[2];
  for (int i = 0; i < 2; ++i) cost[i] = 256 * a.side[i].steps + rot;
  int64_t budget = (T * (cost[0] + cost[1]) + ctas - 1) / ctas;          // of a CTA
  if (budget < 256 * kQkWarps) budget = 256 * kQkWarps;
  for (int i = 0; i < 2; ++i)
    for (int l = 0; l < K; ++l)
      r.first[i * K + l + 1] = r.first[i * K + l] + (int32_t)(((rows[l + 1] - rows[l]) * cost[i] + budget - 1) / budget);
  for (int l = 0; l <= K; ++l) r.rows[l] = rows[l];
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int grid = r.first[2 * K];
  if (grid > 0) {
    void* list[] = {&a, &r};
    if (launch_behind(fn, dim3(grid), dim3(kQkThreads), list, 0, s, true) != cudaSuccess) return BKMOO_ERR_CUDA;
  }
  if (!weights) return BKMOO_OK;
  QkWeightGrads v = {};
  for (int l = 0; l < K; ++l) {
    v.dw[l] = dw_q[l];
    v.dw[K + l] = dw_k[l];
  }
  for (int i = 0; i <= 2 * K; ++i) v.first[i] = r.first[i];
  v.part = r.part;
  v.hd = a.hd;
  v.f32 = dw_dtype == BKMOO_F32;
  v.accumulate = accumulate;
  void* list[] = {&v};
  return launch_behind((const void*)qk_weight_kernel, dim3(2 * K, (a.hd + 31) / 32), dim3(1024), list, 0, s, true) ==
                 cudaSuccess
             ? BKMOO_OK
             : BKMOO_ERR_CUDA;
}
