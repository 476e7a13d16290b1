// Log probabilities of given tokens under rows of logits, with the rows' entropy and
// their most likely tokens, and the gradient of the logits (include/bkmoo.h).
//
// One pass over the logits with a running maximum m, s = sum e^(z - m) and, for the
// entropy, u = sum e^(z - m) (z - m): when the maximum rises by d, s becomes e^-d s and u
// e^-d (u - d s).  Then log p_v = z_v - m - log s, and H = log s - u / s, a sum of two
// terms that are not negative.  Bound by memory: a row is read once.
//
// The n most likely tokens need no second pass over the row: the n-th largest of the
// threads' maxima is a bound that at least n elements reach, and the elements that reach
// it lie with the threads whose maximum does, n of them unless there are ties.
#include <math.h>

#include "row_ops.cuh"
#include "tensor_core.cuh"

namespace bkmoo {
namespace {

constexpr int kLogpThreads = 256;
constexpr int kLogpWarps = kLogpThreads / 32;
constexpr int kMaxTop = 32;
constexpr int kMaxCluster = 8;
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

// m, s and u of a set of logits, u in units of log2.
struct Sums {
  float m, s, u;
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
// a and b of two disjoint sets.
template <bool ENTROPY>
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b) {
  Sums r;
  r.m = fmaxf(a.m, b.m);
  const float at = base_of(r.m);
  // a set without a finite logit has s = 0; minus infinity less a finite number would do for
  // 2^x but not for u
  const float da = fmaxf((a.m - at) * kLog2e, kLowest), db = fmaxf((b.m - at) * kLog2e, kLowest);
  const float ea = exp2f(da), eb = exp2f(db);
  r.s = a.s * ea + b.s * eb;
  r.u = ENTROPY ? ea * fmaf(da, a.s, a.u) + eb * fmaf(db, b.s, b.u) : 0.0f;
  return r;
}
template <bool ENTROPY, int N>
__device__ __forceinline__ void take(Sums& r, const float (&z)[N]) {
  float top = z[0];
#pragma unroll
  for (int j = 1; j < N; ++j) top = fmaxf(top, z[j]);
  if (top > r.m) {
    const float d = fmaxf((r.m - top) * kLog2e, kLowest), e = exp2f(d);
    if (ENTROPY) r.u = e * fmaf(d, r.s, r.u);
    r.s *= e;
    r.m = top;
  }
  const float at = base_of(r.m);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float x = (z[j] - at) * kLog2e, e = exp2f(x);
    r.s += e;
    if (ENTROPY) r.u = fmaf(e, fmaxf(x, kLowest), r.u);
  }
}

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
// The single element of thread t, if it has one: (value, column).
template <class E>
__device__ __forceinline__ int single_at(const Part<E>& p, int t) {
  if (p.front && t < p.head) return t;
  if (p.back && t >= 16 && t < 16 + p.tail) return p.body + p.vecs * kVec<E> + t - 16;
  return -1;
}

template <class E>
constexpr int kBuffer = kMaxTop + kLogpThreads * kVec<E>;

// The n first of buffer[0..count) in order into list, zeros behind them; count may be less.
__device__ void first_of(const uint64_t* buffer, int count, int n, uint64_t* list) {
  for (int i = threadIdx.x; i < n; i += kLogpThreads)
    if (i >= count) list[i] = 0;
  for (int i = threadIdx.x; i < count; i += kLogpThreads) {
    const uint64_t mine = buffer[i];
    int before = 0;
    for (int j = 0; j < count; ++j) before += buffer[j] > mine;
    if (before < n) list[before] = mine;
  }
}

template <class E>
struct TopRoom {
  uint64_t buffer[kBuffer<E>];
  uint64_t list[kMaxTop];
  uint64_t merged[kMaxTop * kMaxCluster];
  uint32_t best[kLogpThreads];
  int16_t who[kLogpThreads];
  int candidates, count;
  uint32_t bound;
};

// list: the n first places of this CTA's part, given every thread's maximum.
template <class E>
__device__ void top_of_part(const Part<E>& p, float m, int n, TopRoom<E>& t) {
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  // (a thread without a finite maximum may have nothing but NaN, which is below all)
  t.best[tid] = m > -INFINITY ? ordered(m) : 0u;
  if (tid == 0) t.candidates = t.count = 0;
  __syncthreads();
  if (wid == 0) {
    // the n-th largest of the maxima, its low half dropped: 16 halvings
    uint32_t mine[kLogpThreads / 32];
#pragma unroll
    for (int j = 0; j < kLogpThreads / 32; ++j) mine[j] = t.best[lane + 32 * j] >> 16;
    uint32_t bound = 0;
    for (uint32_t bit = 0x8000u; bit != 0; bit >>= 1) {
      int reach = 0;
#pragma unroll
      for (int j = 0; j < kLogpThreads / 32; ++j) reach += mine[j] >= (bound | bit);
      if (__reduce_add_sync(0xffffffffu, reach) >= n) bound |= bit;
    }
    if (lane == 0) t.bound = bound << 16;
  }
  __syncthreads();
  const uint32_t bound = t.bound;
  if (t.best[tid] >= bound) t.who[atomicAdd(&t.candidates, 1)] = (int16_t)tid;
  auto keep = [&](float z, int v) {
    if (ordered(z) >= bound) {
      const int at = atomicAdd(&t.count, 1);
      if (at < kBuffer<E>) t.buffer[at] = place_of(z, v);
    }
  };
  const int single = single_at(p, tid);
  if (single >= 0) keep(widen(p.row[single]), single);
  __syncthreads();
  const int candidates = t.candidates;
  for (int c = wid; c < candidates; c += kLogpWarps) {
    for (int i = p.first + t.who[c] + lane * kLogpThreads; i < p.last; i += 32 * kLogpThreads) {
      float z[kVec<E>];
      unpack(vector_at(p, i), z);
#pragma unroll
      for (int j = 0; j < kVec<E>; ++j) keep(z[j], p.body + i * kVec<E> + j);
    }
  }
  __syncthreads();
  if (t.count <= kBuffer<E>) {
    first_of(t.buffer, t.count, n, t.list);
    return;
  }
  // More elements reach the bound than there is room for (equal logits, or the best ones
  // with a few threads): stripe by stripe, keeping the n first so far.
  __syncthreads();
  if (tid == 0) t.count = 0;
  uint64_t least = 0;                   // the n-th place so far
  __syncthreads();
  auto better = [&](float z, int v) {
    const uint64_t at = place_of(z, v);
    if (at > least) t.buffer[atomicAdd(&t.count, 1)] = at;
  };
  for (int from = p.first - kLogpThreads; from < p.last; from += kLogpThreads) {
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
      first_of(t.buffer, count, n, t.list);
      __syncthreads();
      least = t.list[n - 1];
      for (int i = tid; i < n; i += kLogpThreads) t.buffer[i] = t.list[i];
      if (tid == 0) t.count = n;
    }
    __syncthreads();
  }
  first_of(t.buffer, t.count, n, t.list);
}

__device__ __forceinline__ Sums sums_at(const Sums* p, unsigned rank) {
  const uint32_t at = peer_smem(p, rank);
  Sums r;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(r.m) : "r"(at) : "memory");
  asm volatile("ld.shared::cluster.f32 %0, [%1 + 4];" : "=f"(r.s) : "r"(at) : "memory");
  asm volatile("ld.shared::cluster.f32 %0, [%1 + 8];" : "=f"(r.u) : "r"(at) : "memory");
  return r;
}
__device__ __forceinline__ uint64_t word_at(const uint64_t* p, unsigned rank) {
  uint64_t r;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(r) : "r"(peer_smem(p, rank)) : "memory");
  return r;
}

// A row by a cluster of CTAs (one, two, four or eight), each a part of it.
template <class E, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(kLogpThreads) token_logp_kernel(const LogpArgs a, const int parts) {
  grid_wait();
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const unsigned rank = parts > 1 ? cluster_rank() : 0;
  const int64_t t = blockIdx.x / (unsigned)parts;
  const Part<E> p = part_of(static_cast<const E*>(a.logits) + t * a.ld, a.V, rank, parts);
  Sums r = {-INFINITY, 0.0f, 0.0f};
  constexpr int kAhead = 4;
  int i = p.first + tid;
  for (; i + (kAhead - 1) * kLogpThreads < p.last; i += kAhead * kLogpThreads) {
    uint4 v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) v[j] = vector_at(p, i + j * kLogpThreads);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      float z[kVec<E>];
      unpack(v[j], z);
      take<ENTROPY>(r, z);
    }
  }
  for (; i < p.last; i += kLogpThreads) {
    float z[kVec<E>];
    unpack(vector_at(p, i), z);
    take<ENTROPY>(r, z);
  }
  const int single = single_at(p, tid);
  if (single >= 0) {
    const float z[1] = {widen(p.row[single])};
    take<ENTROPY>(r, z);
  }
  const float best = r.m;
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) {
    const Sums o = {__shfl_xor_sync(0xffffffffu, r.m, w), __shfl_xor_sync(0xffffffffu, r.s, w),
                    ENTROPY ? __shfl_xor_sync(0xffffffffu, r.u, w) : 0.0f};
    // the lower lane first, so that both come to the same sum
    r = (lane & w) ? join<ENTROPY>(o, r) : join<ENTROPY>(r, o);
  }
  __shared__ Sums warps[kLogpWarps];
  __shared__ Sums whole;
  if (lane == 0) warps[wid] = r;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kLogpWarps; ++w) r = join<ENTROPY>(r, warps[w]);
    whole = r;
  }
  extern __shared__ __align__(16) unsigned char room[];
  TopRoom<E>& top = *reinterpret_cast<TopRoom<E>*>(room);
  if (TOP) top_of_part(p, best, a.n_top, top);
  if (parts > 1) {
    cluster_sync();                       // the others' sums and lists are there
    if (rank == 0) {
      if (tid == 0) {
        Sums all = whole;
        for (int k = 1; k < parts; ++k) all = join<ENTROPY>(all, sums_at(&whole, k));
        r = all;
      }
      if (TOP)
        for (int j = tid; j < parts * a.n_top; j += kLogpThreads)
          top.merged[j] = word_at(&top.list[j % a.n_top], j / a.n_top);
    }
    cluster_sync();                       // they have been read
    if (rank != 0) return;
    if (tid == 0) whole = r;
    if (TOP) first_of(top.merged, parts * a.n_top, a.n_top, top.list);
  }
  __syncthreads();
  const float m = whole.m, L = logf(whole.s);
  const bool empty = whole.s == 0.0f;   // nothing but minus infinity (a finite maximum adds 1, NaN NaN)
  if (tid == 0) {
    if (a.stats) a.stats[t] = make_float2(m, L);
    const int64_t v = load_id(a.targets, a.id_bytes, t);
    float out = 0.0f;
    if (v >= 0 && v < a.V) out = empty ? -INFINITY : widen(p.row[v]) - m - L;
    a.logp[t] = out;
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
template <class E>
constexpr int kGradPiece = kLogpThreads * kGradVecs * kVec<E>;

// dz_v = g ([v = target] - p_v) - h p_v (log p_v + H).  Bound by memory: a row is read and
// written once.  A row whose g and h are 0 is not read.
template <class E, bool ENTROPY>
__global__ void __launch_bounds__(kLogpThreads) token_logp_grad_kernel(const LogpGradArgs a) {
  grid_wait();
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
    const int i0 = piece * kLogpThreads * kGradVecs + tid;
    uint4* to = reinterpret_cast<uint4*>(out + p.body);
    uint4 x[kGradVecs];
    if (!none) {
#pragma unroll
      for (int j = 0; j < kGradVecs; ++j)
        if (i0 + j * kLogpThreads < p.vecs) x[j] = vector_at(p, i0 + j * kLogpThreads);
    }
#pragma unroll
    for (int j = 0; j < kGradVecs; ++j) {
      const int i = i0 + j * kLogpThreads;
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
    for (int v = piece * kGradPiece<E> + tid, k = 0; k < kGradVecs * kVec<E> && v < a.V; ++k, v += kLogpThreads)
      out[v] = narrow<E>(none ? 0.0f : grad(widen(row[v]), v));
  }
}

template <class E>
const void* logp_fn(bool entropy, bool top) {
  return entropy ? top ? (const void*)token_logp_kernel<E, true, true> : (const void*)token_logp_kernel<E, true, false>
         : top   ? (const void*)token_logp_kernel<E, false, true>
                 : (const void*)token_logp_kernel<E, false, false>;
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
  int parts = 1;
  while (parts < kMaxCluster && T * parts * 2 <= 8 * sms && V / (2 * parts) >= 4096) parts *= 2;
  if (T * parts > 0x7fffffffll) return BKMOO_ERR_INVALID;
  LogpArgs a = {logits, ld, T, (int32_t)V, targets, id_bytes, n_top, logp,
                reinterpret_cast<float2*>(stats), entropy, top_ids, top_logp};
  const bool f32 = dtype == BKMOO_F32;
  const void* fn = f32 ? logp_fn<float>(entropy, n_top > 0) : logp_fn<__nv_bfloat16>(entropy, n_top > 0);
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
  cfg.blockDim = dim3(kLogpThreads);
  cfg.dynamicSmemBytes = n_top == 0 ? 0 : f32 ? sizeof(TopRoom<float>) : sizeof(TopRoom<__nv_bfloat16>);
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
  const int64_t piece = f32 ? kGradPiece<float> : kGradPiece<__nv_bfloat16>;
  const int64_t pieces = (V + piece - 1) / piece;
  if (T * pieces > 0x7fffffffll) return BKMOO_ERR_INVALID;
  LogpGradArgs a = {logits, d_logits, ld, ld_d, (int32_t)V, targets, id_bytes,
                    reinterpret_cast<const float2*>(stats), d_logp, d_entropy, entropy, (uint32_t)pieces};
  const void* fn = f32 ? d_entropy ? (const void*)token_logp_grad_kernel<float, true>
                                   : (const void*)token_logp_grad_kernel<float, false>
                   : d_entropy ? (const void*)token_logp_grad_kernel<__nv_bfloat16, true>
                               : (const void*)token_logp_grad_kernel<__nv_bfloat16, false>;
  void* list[] = {&a};
  return launch_behind(fn, dim3((unsigned)(T * pieces)), dim3(kLogpThreads), list, 0,
                       static_cast<cudaStream_t>(stream), true) == cudaSuccess
             ? BKMOO_OK
             : BKMOO_ERR_CUDA;
}
