// Log probabilities of given tokens under rows of logits, with the rows' entropy and
// their most likely tokens, and the gradient of the logits (include/bkmoo.h).
//
// One pass over the logits with a running maximum m, s = sum e^(z - m) and, for the
// entropy, u = sum e^(z - m) (z - m): when the maximum rises by d, s becomes e^-d s and u
// e^-d (u - d s).  Then log p_v = z_v - m - log s, and H = log s - u / s, a sum of two
// terms that are not negative.  Bound by memory: a row is read once.
//
// The n most likely tokens need no second pass over the row: each warp gives the q-th largest
// of its threads' maxima, q its share of n, so n elements at least reach the least of these.
// The elements that do lie in a few threads' best batches of vectors, which are read again
// (a thread whose second batch reaches it too has all of its own read again).
#include <math.h>

#include "row_ops.cuh"
#include "tensor_core.cuh"

namespace bkmoo {
namespace {

constexpr int kMaxTop = 32;
constexpr int kMaxCluster = 8;
constexpr int kAhead = 4;               // vectors of a thread that are on their way at once
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// (z - m) log2(e) below this counts as this where it is multiplied by 2^itself: 2^-1000 is 0
// and 0 times minus infinity would not be.
constexpr float kLowest = -1000.0f;

struct LogpArgs {
  const void* logits;
  int64_t ld;
  int64_t T;
  int32_t V;
  const void* targets;
  int32_t id_bytes;
  int32_t n_top;
  float* logp;
  float2* stats;
  float* entropy;
  int64_t* top_ids;
  float* top_logp;
};

// A value as a whole number of the same order, NaN below all; equal values (0 and -0 among
// them) give equal numbers.
__device__ __forceinline__ uint32_t ordered(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return z != z ? 1u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return o == 1u ? __uint_as_float(0x7fc00000u) : __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
// The order of (value, index): the larger value first, then the lower index.  Never 0.
__device__ __forceinline__ uint64_t place_of(float z, int v) { return (uint64_t)ordered(z) << 32 | (uint32_t)~v; }

// m, s and u of a set of logits, u in units of log2.
struct Sums {
  float m, s, u;
};
// 2^x by one instruction, off by 2^-22 of itself; 0 below 2^-126.
__device__ __forceinline__ float pow2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
// The sets of a warp's first W lanes (the others hold none), their sums in the lanes' order: all
// to the largest maximum first, then plain sums.
template <bool ENTROPY, int W>
__device__ __forceinline__ Sums join_lanes(Sums r) {
  const float m = value_of(__reduce_max_sync(0xffffffffu, ordered(r.m)));
  // a set without a finite logit has s = 0; minus infinity less a finite number would do for
  // 2^x but not for u
  const float d = fmaxf((r.m - base_of(m)) * kLog2e, kLowest), e = pow2(d);
  if (ENTROPY) r.u = e * fmaf(d, r.s, r.u);
  r.s *= e;
  r.m = m;
#pragma unroll
  for (int w = 1; w < W; w *= 2) {
    r.s += __shfl_xor_sync(0xffffffffu, r.s, w);
    if (ENTROPY) r.u += __shfl_xor_sync(0xffffffffu, r.u, w);
  }
  return r;
}
// A new maximum, if `top` is one.
template <bool ENTROPY>
__device__ __forceinline__ bool raise(Sums& r, float top) {
  if (!(top > r.m)) return false;
  const float d = fmaxf((r.m - top) * kLog2e, kLowest), e = pow2(d);
  if (ENTROPY) r.u = e * fmaf(d, r.s, r.u);
  r.s *= e;
  r.m = top;
  return true;
}
// z, none of them above the maximum.
template <bool ENTROPY, int N>
__device__ __forceinline__ void take(Sums& r, const float (&z)[N]) {
  const float at = base_of(r.m);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float x = (z[j] - at) * kLog2e, e = pow2(x);
    r.s += e;
    if (ENTROPY) r.u = fmaf(e, fmaxf(x, kLowest), r.u);
  }
}
// Where a thread has more than kLongBatches batches of a row (2048 bf16 logits, 1024 fp32 ones), its sums
// so far are put aside after as many, and begin again: in one fp32 sum of n terms each of them may be off
// by n 2^-24 of itself, and all to the same side where the logits are alike.  A row of 2^27 fp32 logits
// of two values was 9e-4 off in log s.  A kernel of its own: 600 bf16 rows of 2^21 take 425 us with it and
// 417 without, and the same steps in the kernel for the other rows cost those 1%.
constexpr int kLongBatches = 64;
constexpr int kLongVecs = kLongBatches * kAhead * 256;       // of a CTA
template <bool ENTROPY>
__device__ __forceinline__ void put_aside(Sums& r, Sums& aside) {
  raise<ENTROPY>(aside, r.m);            // (r's maximum is never the lower one)
  aside.s += r.s;
  if (ENTROPY) aside.u += r.u;
  r.s = r.u = 0.0f;
}
// The largest of a vector, NaN aside.
__device__ __forceinline__ float largest(const uint4& v, float) {
  return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
}
__device__ __forceinline__ float largest(const uint4& v, __nv_bfloat16) {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
  const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
  return fmaxf(__low2float(m), __high2float(m));
}
// Columns of a row's part: elements ahead of the first whole 16-byte vector and behind the
// last by thread, vectors in between.
template <class E>
struct Part {
  const E* row;
  int head, body, vecs, tail;          // elements, first column of the vectors, vectors, elements
  int first, last;                     // this CTA's vectors
  bool front, back;                    // it has the head, the tail
};
template <class E>
__device__ __forceinline__ Part<E> part_of(const E* row, int V, unsigned rank, unsigned parts) {
  Part<E> p;
  p.row = row;
  const int ahead = (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(E);
  p.head = ahead < V ? ahead : V;
  p.body = p.head;
  p.vecs = (V - p.head) / kVec<E>;
  p.tail = V - p.head - p.vecs * kVec<E>;
  const int each = (p.vecs + (int)parts - 1) / (int)parts;
  p.first = min((int)rank * each, p.vecs);
  p.last = min(p.first + each, p.vecs);
  p.front = rank == 0;
  p.back = rank == parts - 1;
  return p;
}
template <class E>
__device__ __forceinline__ uint4 vector_at(const Part<E>& p, int i) {
  return __ldcg(reinterpret_cast<const uint4*>(p.row + p.body) + i);
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) {
  return i < 2 ? i == 0 ? v.x : v.y : i == 2 ? v.z : v.w;
}
__device__ __forceinline__ float element(const uint4& v, int e, float) { return __uint_as_float(word(v, e)); }
__device__ __forceinline__ float element(const uint4& v, int e, __nv_bfloat16) {
  const uint32_t w = word(v, e / 2);
  return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
}
// The single element of thread t, if it has one: (value, column).
template <class E>
__device__ __forceinline__ int single_at(const Part<E>& p, int t) {
  if (p.front && t < p.head) return t;
  if (p.back && t >= 16 && t < 16 + p.tail) return p.body + p.vecs * kVec<E> + t - 16;
  return -1;
}

template <class E, int N>
constexpr int kBuffer = kMaxTop + N * kVec<E>;
constexpr int kScan = 64;               // elements that first_of looks at in a step

// The n first of buffer[0..count) in order into list, zeros behind them; 4 threads an element.
// The buffer's memory goes on to the next multiple of kScan.
template <int N>
__device__ void first_of(const uint64_t* buffer, int count, int n, uint64_t* list) {
  const int sub = threadIdx.x % 4;
  for (int i = count + threadIdx.x; i < n; i += N) list[i] = 0;
  for (int i0 = 0; i0 < count; i0 += N / 4) {
    const int i = i0 + threadIdx.x / 4;
    const uint64_t mine = i < count ? buffer[i] : ~0ull;
    int before = 0;
    for (int j0 = 0; j0 < count; j0 += kScan) {
#pragma unroll
      for (int k = 0; k < kScan / 8; ++k) {
        const int j = j0 + 8 * k + 2 * sub;
        const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(buffer + j);
        before += (j < count && v.x > mine) + (j + 1 < count && v.y > mine);
      }
    }
#pragma unroll
    for (int w = 1; w < 4; w *= 2) before += __shfl_xor_sync(0xffffffffu, before, w);
    if (sub == 0 && i < count && before < n) list[before] = mine;
  }
}

template <class E, int N>
struct TopRoom {
  alignas(16) uint64_t buffer[(kBuffer<E, N> + kScan - 1) / kScan * kScan];
  uint64_t list[kMaxTop];
  uint64_t merged[kMaxTop * kMaxCluster];       // the cluster's lists
  int near[N], who[N];                  // threads of which one batch is looked at again, all of them
  int n_near, n_who, count;
  uint32_t bounds[N / 32];
};

// The largest of a thread's vectors, its batch of kAhead (by its first vector), and the largest
// of the other batches.
struct Best {
  float first, second;
  int at;
};
// list: the n first places of this CTA's part.
template <class E, int N>
__device__ void top_of_part(const Part<E>& p, const Best& mine, int n, TopRoom<E, N>& t) {
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  constexpr int kWarpsHere = N / 32;
  // (a thread without a finite maximum may have nothing but NaN, which is below all)
  const uint32_t best = mine.first > -INFINITY ? ordered(mine.first) : 0u;
  const uint32_t other = mine.second > -INFINITY ? ordered(mine.second) : 0u;
  if (tid == 0) t.n_near = t.n_who = t.count = 0;
  // Each warp's q-th largest maximum, q its share of n among the warps that have a vector for
  // every lane: n maxima at least reach the least of these.
  const int full = min(kWarpsHere, (p.last - p.first) / 32);
  uint32_t left = best, share = 0;
  for (int q = full > 0 ? (n + full - 1) / full : 0; q > 0;) {
    share = __reduce_max_sync(0xffffffffu, left);
    if (share == 0) break;
    const bool it = left == share;
    q -= __popc(__ballot_sync(0xffffffffu, it));
    if (it) left = 0;
  }
  if (lane == 0) t.bounds[wid] = share;
  __syncthreads();
  uint32_t bound = t.bounds[0];
#pragma unroll
  for (int w = 1; w < kWarpsHere; ++w)
    if (w < full) bound = min(bound, t.bounds[w]);
  auto note = [&](bool it, int* list, int* n, int what) {
    const uint32_t those = __ballot_sync(0xffffffffu, it);
    int at = 0;
    if (those == 0) return;
    if (lane == 0) at = atomicAdd(n, __popc(those));
    at = __shfl_sync(0xffffffffu, at, 0) + __popc(those & ((1u << lane) - 1));
    if (it) list[at] = what;
  };
  const uint32_t reach = max(bound, 1u);
  note(best >= reach && other < reach, t.near, &t.n_near, mine.at);
  note(best >= reach && other >= reach, t.who, &t.n_who, p.first + tid);
  // Elements from the bound up; where they are more than there is room for (many as large as the
  // bound), or the bound is minus infinity, those above it.
  const float low = bound == 0 ? -INFINITY : value_of(bound);
  bool above = bound == 0;
  auto keep = [&](uint32_t those, const auto& z, int v) {
    int at = atomicAdd(&t.count, __popc(those));
    for (; those; those &= those - 1, ++at)
      if (at < kBuffer<E, N>) t.buffer[at] = place_of(z(__ffs(those) - 1), v + __ffs(those) - 1);
  };
  const int single = single_at(p, tid);
  for (;;) {
    auto reaches = [&](float z) { return above ? z > low : z >= low; };
    if (single >= 0) {
      const float z = widen(p.row[single]);
      if (reaches(z)) keep(1u, [&](int) { return z; }, single);
    }
    __syncthreads();
    // those threads' vectors, by all threads
    const int near = kAhead * t.n_near, whole = t.n_who;
    const int items = near + whole * ((p.last - p.first + N - 1) / N);
    for (int i0 = tid; i0 < items; i0 += kAhead * N) {
      uint4 x[kAhead];
      int at[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k * N;
        at[k] = p.last;
        if (i >= items) continue;
        if (i < near) {
          at[k] = t.near[i / kAhead] + i % kAhead * N;
        } else {
          const int j = (i - near) / whole;
          at[k] = t.who[i - near - j * whole] + j * N;
        }
        if (at[k] < p.last) x[k] = vector_at(p, at[k]);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (at[k] >= p.last) continue;
        float z[kVec<E>];
        unpack(x[k], z);
        uint32_t those = 0;
#pragma unroll
        for (int e = 0; e < kVec<E>; ++e) those |= reaches(z[e]) ? 1u << e : 0u;
        // (the elements by their number from the words: an index into registers is none)
        if (those) keep(those, [&](int e) { return element(x[k], e, E()); }, p.body + at[k] * kVec<E>);
      }
    }
    __syncthreads();
    if (above || t.count <= kBuffer<E, N>) break;
    __syncthreads();
    above = true;
    if (tid == 0) t.count = 0;
    __syncthreads();
  }
  int have = t.count;
  if (have <= kBuffer<E, N>) {
    first_of<N>(t.buffer, have, n, t.list);
    if (have >= n) return;
    // the others are as large as the bound, or NaN: the first ones of the row
    const int end = p.back ? p.body + p.vecs * kVec<E> + p.tail : p.body + p.last * kVec<E>;
    for (int nan = 0; nan < 2 && have < n; ++nan) {
      for (int v0 = p.front ? 0 : p.body + p.first * kVec<E>; v0 < end && have < n; v0 += N) {
        const bool in = v0 + tid < end;
        const float z = in ? widen(p.row[v0 + tid]) : 0.0f;
        const uint32_t those = __ballot_sync(0xffffffffu, in && (nan ? z != z : z == low));
        __syncthreads();
        if (lane == 0) t.near[wid] = __popc(those);
        __syncthreads();
        int at = have;
        for (int w = 0; w < kWarpsHere; ++w) {
          if (w < wid) at += t.near[w];
          have += t.near[w];
        }
        at += __popc(those & ((1u << lane) - 1));
        if ((those >> lane & 1) && at < n) t.list[at] = place_of(z, v0 + tid);
      }
    }
    return;
  }
  // More elements than there is room for all the same (the best ones lie with a few threads):
  // stripe by stripe, keeping the n first so far.
  __syncthreads();
  if (tid == 0) t.count = 0;
  uint64_t least = 0;                   // the n-th place so far
  __syncthreads();
  auto better = [&](float z, int v) {
    const uint64_t at = place_of(z, v);
    if (at > least) t.buffer[atomicAdd(&t.count, 1)] = at;
  };
  for (int from = p.first - N; from < p.last; from += N) {
    if (from < p.first) {
      if (single >= 0) better(widen(p.row[single]), single);
    } else if (from + tid < p.last) {
      float z[kVec<E>];
      unpack(vector_at(p, from + tid), z);
#pragma unroll
      for (int j = 0; j < kVec<E>; ++j) better(z[j], p.body + (from + tid) * kVec<E> + j);
    }
    __syncthreads();
    const int count = t.count;
    if (count > n) {
      first_of<N>(t.buffer, count, n, t.list);
      __syncthreads();
      least = t.list[n - 1];
      for (int i = tid; i < n; i += N) t.buffer[i] = t.list[i];
      if (tid == 0) t.count = n;
    }
    __syncthreads();
  }
  first_of<N>(t.buffer, t.count, n, t.list);
}

// Writes to shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ void put_sums(const Sums* p, unsigned rank, const Sums& v) {
  const uint32_t at = peer_smem(p, rank);
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v.m) : "memory");
  asm volatile("st.shared::cluster.f32 [%0 + 4], %1;" ::"r"(at), "f"(v.s) : "memory");
  asm volatile("st.shared::cluster.f32 [%0 + 8], %1;" ::"r"(at), "f"(v.u) : "memory");
}
__device__ __forceinline__ void put_word(const uint64_t* p, unsigned rank, uint64_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(peer_smem(p, rank)), "l"(v) : "memory");
}
// The halves of a barrier over the cluster.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// A row by a cluster of CTAs (one, two, four or eight), each a part of it.  Memory-bound: 8192 x
// 128256 bf16 291 to 295 us (7.2 TB/s), with the entropy 299, with the 20 likeliest too 353; 1531 x
// 50257 fp32 51, 49 and 59 us.  One row of 151936 takes 3.8 us and 7, a chain of latencies.
// 6 CTAs of 256 to an SM leave 40 registers (of fp32 with entropy and likeliest 12 bytes go to memory):
// at 5, 1531 rows are two rounds and a little.
template <class E, bool ENTROPY, bool TOP, int N, bool LONG = false>
__global__ void __launch_bounds__(N, N == 32 ? 32 : 1536 / N) token_logp_kernel(const LogpArgs a, const int parts) {
  grid_wait();
  grid_release();
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const unsigned rank = parts > 1 ? cluster_rank() : 0;
  if (parts > 1) cluster_arrive();
  const int64_t t = blockIdx.x / (unsigned)parts;
  const Part<E> p = part_of(static_cast<const E*>(a.logits) + t * a.ld, a.V, rank, parts);
  const int64_t target = load_id(a.targets, a.id_bytes, t);
  Sums r = {-INFINITY, 0.0f, 0.0f};
  Best best = {-INFINITY, -INFINITY, p.first + tid};
  auto batches = [&](int i0, int end) {
    for (int i = i0; i < end; i += kAhead * N) {
      uint4 v[kAhead];
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j * N < p.last) v[j] = vector_at(p, i + j * N);
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j * N < p.last) top = fmaxf(top, largest(v[j], E()));
      const float old = r.m;
      if (raise<ENTROPY>(r, top)) {
        if (TOP) best.second = old, best.at = i;
      } else if (TOP) {
        best.second = fmaxf(best.second, top);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (i + j * N >= p.last) break;
        float z[kVec<E>];
        unpack(v[j], z);
        take<ENTROPY>(r, z);
      }
    }
  };
  if (LONG) {
    __shared__ Sums aside[N];
    aside[tid] = r;
    for (int from = p.first; from < p.last; from += kLongVecs) {
      batches(from + tid, min(from + kLongVecs, p.last));
      put_aside<ENTROPY>(r, aside[tid]);
    }
    r = aside[tid];
  } else {
    batches(p.first + tid, p.last);
  }
  best.first = r.m;
  const int single = single_at(p, tid);
  if (single >= 0) {
    const float z[1] = {widen(p.row[single])};
    raise<ENTROPY>(r, z[0]);
    take<ENTROPY>(r, z);
  }
  const bool has = target >= 0 && target < a.V;
  const E z_target = tid == 0 && has ? p.row[target] : narrow<E>(0.0f);
  r = join_lanes<ENTROPY, 32>(r);
  constexpr int kWarpsHere = N / 32;
  const Sums nothing = {-INFINITY, 0.0f, 0.0f};
  __shared__ Sums warps[kWarpsHere];
  __shared__ Sums whole;
  if (lane == 0) warps[wid] = r;
  __syncthreads();
  if (wid == 0) {
    r = join_lanes<ENTROPY, kWarpsHere>(lane < kWarpsHere ? warps[lane] : nothing);
    if (lane == 0) whole = r;
  }
  extern __shared__ __align__(16) unsigned char room[];
  TopRoom<E, N>& top = *reinterpret_cast<TopRoom<E, N>*>(room);
  if (TOP) top_of_part(p, best, a.n_top, top);
  if (parts > 1) {
    // to the first CTA, all of which have begun by now
    __shared__ Sums peers[kMaxCluster];
    __syncthreads();
    cluster_wait();
    if (TOP && tid == 0) top.count = 0;     // (after the last use of it, ahead of the barrier below)
    if (TOP && tid < a.n_top) put_word(&top.merged[rank * a.n_top + tid], 0, top.list[tid]);
    if (tid == 0) put_sums(&peers[rank], 0, whole);
    cluster_sync();
    if (rank != 0) return;
    if (wid == 0) {
      r = join_lanes<ENTROPY, kMaxCluster>(lane < parts ? peers[lane] : nothing);
      if (lane == 0) whole = r;
    }
    if (TOP) {
      // at least n_top of the lists' elements are no lower than the lowest of their q-th ones
      const int n = a.n_top, q = (n + parts - 1) / parts;
      uint64_t least = ~0ull;
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k)
        if (k < parts) least = min(least, top.merged[k * n + q - 1]);
      for (int i = tid; i < parts * n; i += N) {
        const uint64_t v = top.merged[i];
        if (v >= least) top.buffer[atomicAdd(&top.count, 1)] = v;
      }
      __syncthreads();
      first_of<N>(top.buffer, top.count, n, top.list);
    }
  }
  __syncthreads();
  const float m = whole.m, L = logf(whole.s);
  const bool empty = whole.s == 0.0f;   // nothing but minus infinity (a finite maximum adds 1, NaN NaN)
  if (tid == 0) {
    if (a.stats) a.stats[t] = make_float2(m, L);
    a.logp[t] = !has ? 0.0f : empty ? -INFINITY : widen(z_target) - m - L;
    if (ENTROPY) a.entropy[t] = empty ? 0.0f : L - whole.u / whole.s * kLn2;
  }
  if (TOP && tid < a.n_top) {
    const uint64_t place = top.list[tid];
    const float z = value_of((uint32_t)(place >> 32));
    a.top_ids[t * a.n_top + tid] = (int64_t)(uint32_t)~(uint32_t)place;
    a.top_logp[t * a.n_top + tid] = empty ? -INFINITY : z - m - L;
  }
}

struct LogpGradArgs {
  const void* logits;
  void* out;
  int64_t ld, ld_out;
  int32_t V;
  const void* targets;
  int32_t id_bytes;
  const float2* stats;
  const float *g, *h, *entropy;
  uint32_t pieces;                       // of a row
};
constexpr int kGradVecs = 4;             // of a thread
template <class E, int N>
constexpr int kGradPiece = N * kGradVecs * kVec<E>;

// dz_v = g ([v = target] - p_v) - h p_v (log p_v + H).  A row is read and written once; one whose g
// and h are 0 is not read.  Bound by memory where a row of the result starts at the same place of
// 16 bytes as the logits': 8192 x 50257 bf16 256 us, 4096 fp32 233.  Others go element by element, a load
// on its way at a time: 702 and 380 us with rows of the result padded to 50264, of which 7 of 8 (fp32:
// 3 of 4) start elsewhere.
template <class E, bool ENTROPY, int N>
__global__ void __launch_bounds__(N) token_logp_grad_kernel(const LogpGradArgs a) {
  grid_wait();
  grid_release();
  const int64_t t = blockIdx.x / a.pieces;
  const int piece = (int)(blockIdx.x % a.pieces);
  const E* row = static_cast<const E*>(a.logits) + t * a.ld;
  E* out = static_cast<E*>(a.out) + t * a.ld_out;
  const int64_t target = load_id(a.targets, a.id_bytes, t);
  // (the log probability of padding is 0 whatever the logits)
  const float g = target < 0 || target >= a.V ? 0.0f : a.g[t];
  const float h = ENTROPY ? a.h[t] : 0.0f, H = ENTROPY ? a.entropy[t] : 0.0f;
  const float2 st = a.stats[t];
  const bool none = (g == 0.0f && h == 0.0f) || st.y == -INFINITY;    // log 0
  auto grad = [&](float z, int v) {
    const float lp = z - st.x - st.y, p = exp2f(lp * kLog2e);
    float d = ENTROPY ? -p * fmaf(h, fmaxf(lp, kLowest) + H, g) : -p * g;
    return v == target ? d + g : d;
  };
  // vectors where both rows start at the same place of 16 bytes
  const bool same = (((uintptr_t)row ^ (uintptr_t)out) & 15) == 0;
  const Part<E> p = part_of(row, a.V, 0, 1);
  const int tid = threadIdx.x;
  if (same) {
    if (piece == 0) {
      const int s = single_at(p, tid);
      if (s >= 0) out[s] = narrow<E>(none ? 0.0f : grad(widen(row[s]), s));
    }
    const int i0 = piece * N * kGradVecs + tid;
    uint4* to = reinterpret_cast<uint4*>(out + p.body);
    uint4 x[kGradVecs];
    if (!none) {
#pragma unroll
      for (int j = 0; j < kGradVecs; ++j)
        if (i0 + j * N < p.vecs) x[j] = vector_at(p, i0 + j * N);
    }
#pragma unroll
    for (int j = 0; j < kGradVecs; ++j) {
      const int i = i0 + j * N;
      if (i >= p.vecs) break;
      if (none) {
        to[i] = make_uint4(0, 0, 0, 0);
        continue;
      }
      float z[kVec<E>];
      unpack(x[j], z);
#pragma unroll
      for (int e = 0; e < kVec<E>; ++e) z[e] = grad(z[e], p.body + i * kVec<E> + e);
      to[i] = repack(z);
    }
  } else {
    for (int v = piece * kGradPiece<E, N> + tid, k = 0; k < kGradVecs * kVec<E> && v < a.V; ++k, v += N)
      out[v] = narrow<E>(none ? 0.0f : grad(widen(row[v]), v));
  }
}

template <class E>
const void* grad_fn(int threads, bool entropy) {
  return threads == 64 ? entropy ? (const void*)token_logp_grad_kernel<E, true, 64> : (const void*)token_logp_grad_kernel<E, false, 64>
         : entropy     ? (const void*)token_logp_grad_kernel<E, true, 256>
                       : (const void*)token_logp_grad_kernel<E, false, 256>;
}
template <class E, int N, bool LONG = false>
const void* logp_fn(bool entropy, bool top) {
  return entropy ? top ? (const void*)token_logp_kernel<E, true, true, N, LONG> : (const void*)token_logp_kernel<E, true, false, N, LONG>
         : top   ? (const void*)token_logp_kernel<E, false, true, N, LONG>
                 : (const void*)token_logp_kernel<E, false, false, N, LONG>;
}
template <class E>
const void* logp_fn(int threads, bool is_long, bool entropy, bool top, size_t* room) {
  *room = !top ? 0 : threads == 32 ? sizeof(TopRoom<E, 32>) : threads == 128 ? sizeof(TopRoom<E, 128>) : sizeof(TopRoom<E, 256>);
  return threads == 32    ? logp_fn<E, 32>(entropy, top)
         : threads == 128 ? logp_fn<E, 128>(entropy, top)
         : is_long        ? logp_fn<E, 256, true>(entropy, top)
                          : logp_fn<E, 256>(entropy, top);
}

bool logits_ok(const void* p, int32_t dtype, int64_t T, int64_t V, int64_t ld) {
  return aligned_at(p, float_bytes(dtype)) && ld >= V && ld <= ((int64_t)1 << 38) && T <= ((int64_t)1 << 31) - 1024;
}

}  // namespace
}  // namespace bkmoo

using namespace bkmoo;

extern "C" int bkmoo_token_logp_forward(const void* logits, int64_t ld, int32_t dtype, int64_t T,
                                        int64_t V, const void* targets, int32_t id_bytes,
                                        float* logp, float* stats, float* entropy, int32_t n_top,
                                        int64_t* top_ids, float* top_logp, void* stream) {
  if (!is_float(dtype) || !is_id(id_bytes) || T < 0 || V < 1 || V > ((int64_t)1 << 30) || n_top < 0 ||
      n_top > kMaxTop || n_top > V)
    return BKMOO_ERR_INVALID;
  if (T == 0) return BKMOO_OK;
  if (!logits_ok(logits, dtype, T, V, ld) || !aligned_at(targets, id_bytes) || !aligned_at(logp, 4) ||
      (stats && !aligned_at(stats, 8)) || (entropy && !aligned_at(entropy, 4)) ||
      (n_top > 0 && (!aligned_at(top_ids, 8) || !aligned_at(top_logp, 4))))
    return BKMOO_ERR_INVALID;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return BKMOO_ERR_CUDA;
  // Few rows: by more CTAs, up to 4 an SM, while each has 4096 logits (200 x 128256 bf16: 11.5 us by
  // one, 9.9 by two, 10.2 by four; 400: 20.5, 19.0 and 19.8, with the 20 likeliest 28, 31 and 35;
  // 1 x 151936: 5.0 by four, 4.0 by eight).
  int parts = 1;
  while (parts < kMaxCluster && T * parts * 2 <= 4 * sms && V / (2 * parts) >= 4096) parts *= 2;
  if (T * parts > 0x7fffffffll) return BKMOO_ERR_INVALID;
  LogpArgs a = {logits, ld, T, (int32_t)V, targets, id_bytes, n_top, logp,
                reinterpret_cast<float2*>(stats), entropy, top_ids, top_logp};
  const bool f32 = dtype == BKMOO_F32;
  const int64_t vecs = V / parts * (int64_t)float_bytes(dtype) / 16;
  // Threads a row (a warp alone, 128 or 256): the fewer, the less of a row's time goes into what
  // its threads do together, but a long row by few is slow.  20000 bf16 rows of 2000: 15, 27 and
  // 45 us, the 20 likeliest 48, 83 and 143; 4096 of 10007: 14, 14.5 and 18 (31, 29, 40); 1500
  // fp32 of 262144: 359, 219 and 240 (750, 273, 256): there 256 is the better choice with the
  // likeliest only, as 1500 rows fit the card once by 128 threads and not by 256, which this does not
  // look at.  Where rows are few, latency counts: 20 rows of 4000 3.2, 2.2 and 2.3 (8.4, 4.5, 4.2).
  const bool many = T * parts >= 8 * sms;
  const int threads = vecs < (many ? 768 : 256) ? 32 : vecs < (many ? 6000 : 1024) ? 128 : 256;
  size_t room = 0;
  const bool is_long = vecs > kLongVecs;
  const void* fn = f32 ? logp_fn<float>(threads, is_long, entropy, n_top > 0, &room)
                       : logp_fn<__nv_bfloat16>(threads, is_long, entropy, n_top > 0, &room);
  void* list[] = {&a, &parts};
  cudaLaunchConfig_t cfg = {};
  // (the kernel waits at its top for the one ahead of it: launch_behind)
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = parts;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(T * parts));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = room;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cfg.attrs = attr;
  cfg.numAttrs = parts > 1 ? 2 : 1;
  return cudaLaunchKernelExC(&cfg, fn, list) == cudaSuccess ? BKMOO_OK : BKMOO_ERR_CUDA;
}

extern "C" int bkmoo_token_logp_backward(const void* logits, int64_t ld, int32_t dtype, int64_t T,
                                         int64_t V, const void* targets, int32_t id_bytes,
                                         const float* stats, const float* entropy,
                                         const float* d_logp, const float* d_entropy,
                                         void* d_logits, int64_t ld_d, void* stream) {
  if (!is_float(dtype) || !is_id(id_bytes) || T < 0 || V < 1 || V > ((int64_t)1 << 30))
    return BKMOO_ERR_INVALID;
  if (T == 0) return BKMOO_OK;
  if (!logits_ok(logits, dtype, T, V, ld) || !logits_ok(d_logits, dtype, T, V, ld_d) ||
      (logits == d_logits && ld != ld_d) || !aligned_at(targets, id_bytes) || !aligned_at(stats, 8) ||
      !aligned_at(d_logp, 4) || (d_entropy && (!aligned_at(d_entropy, 4) || !aligned_at(entropy, 4))))
    return BKMOO_ERR_INVALID;
  const bool f32 = dtype == BKMOO_F32;
  // Short rows go to CTAs of 64 threads, of which more are at work on different rows (20000 bf16 rows
  // of 2000: 28 us, by 256 threads 44; of 8000 98 and 102); long ones to fewer CTAs (8192 rows of
  // 128256: 588 and 544).
  const int threads = V * (int64_t)float_bytes(dtype) / 16 <= 1024 ? 64 : 256;
  const int64_t piece = threads * kGradVecs * (f32 ? kVec<float> : kVec<__nv_bfloat16>);
  const int64_t pieces = (V + piece - 1) / piece;
  if (T * pieces > 0x7fffffffll) return BKMOO_ERR_INVALID;
  LogpGradArgs a = {logits, d_logits, ld, ld_d, (int32_t)V, targets, id_bytes,
                    reinterpret_cast<const float2*>(stats), d_logp, d_entropy, entropy, (uint32_t)pieces};
  const void* fn = f32 ? grad_fn<float>(threads, d_entropy) : grad_fn<__nv_bfloat16>(threads, d_entropy);
  void* list[] = {&a};
  return launch_behind(fn, dim3((unsigned)(T * pieces)), dim3(threads), list, 0,
                       static_cast<cudaStream_t>(stream), true) == cudaSuccess
             ? BKMOO_OK
             : BKMOO_ERR_CUDA;
}
