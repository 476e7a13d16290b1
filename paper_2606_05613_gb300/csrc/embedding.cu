// Rows of an embedding looked up by token and scaled, and the gradient of the embedding
// apart by language (include/bkmoo.h).
//
// Forward: y_t = s W[id_t].  Bound by memory: 16384 rows of 2048 bf16 take 15.3 us (6.3 TB/s), a
// thread with one vector on its way at a time 22.5.
//
// Backward: dW_k[v] = s sum of dy_t over language k's rows t with id_t = v.  The rows are
// put in the order of (language, token, t); then each token's rows lie side by side, and
// a warp sums a piece of 8 to 32 places for 256 columns in that order.  A sum that lies in one
// piece is written (or added) by its warp; the others leave their parts, which are joined in
// the order of the pieces: no atomics on values, the same result every time.  8192 rows of
// 2048 bf16 in 4 languages, added, take 20 us: 9 for the sums, the others a chain of latencies.
//
// The order: 256 rows sorted by a CTA (bitonic, in registers and shared memory), then runs of
// sorted rows merged 32 at a time: a row's place in the merged run is its place in its own
// plus, for each other run, how many there come before it, a binary search.
#include <math.h>

#include "tile_host.cuh"
#include "row_ops.cuh"

namespace bkmoo {
namespace {

constexpr int kEmbedThreads = 256;
constexpr int kSortRun = 256;           // rows that a CTA sorts
constexpr int kMerge = 32;              // runs merged at once
constexpr int kColumns = 256;           // columns of a warp: 8 a lane
constexpr uint32_t kNoToken = 0xffffffffu;

// ---- forward ---------------------------------------------------------------

struct LookupArgs {
  const void *table, *ids;
  void* y;
  int64_t ld, ld_y, T, V;
  int32_t id_bytes;
  uint32_t D, per;                      // columns; pieces of a row: vectors, or kColumns columns
  float scale;
};
// 16 bytes a thread at a time.  A thread has AHEAD of them on their way at once: 4 where there are
// more than the card holds threads.
template <class E, int AHEAD>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const __grid_constant__ LookupArgs a) {
  grid_wait();
  const int64_t n = a.T * a.per;
  for (int64_t i0 = (int64_t)blockIdx.x * (kEmbedThreads * AHEAD) + threadIdx.x; i0 < n;
       i0 += (int64_t)gridDim.x * (kEmbedThreads * AHEAD)) {
    int64_t t[AHEAD], c[AHEAD], id[AHEAD];
    uint4 v[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int64_t i = i0 + j * kEmbedThreads;
      id[j] = -1;
      if (i >= n) continue;
      t[j] = n < (1ll << 32) ? (uint32_t)i / a.per : i / a.per;
      c[j] = (i - t[j] * a.per) * kVec<E>;
      id[j] = load_id(a.ids, a.id_bytes, t[j]);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      v[j] = make_uint4(0, 0, 0, 0);
      if (id[j] >= 0 && id[j] < a.V) v[j] = *reinterpret_cast<const uint4*>(static_cast<const E*>(a.table) + id[j] * a.ld + c[j]);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (i0 + j * kEmbedThreads >= n) break;
      float y[kVec<E>];
      unpack(v[j], y);
#pragma unroll
      for (int e = 0; e < kVec<E>; ++e) y[e] *= a.scale;
      *reinterpret_cast<uint4*>(static_cast<E*>(a.y) + t[j] * a.ld_y + c[j]) = repack(y);
    }
  }
}

// ---- order -----------------------------------------------------------------

// Gradients that are written instead of added to begin as 0.  The kernels of the order, which
// leave most of the card idle, have CTAs for that beside their own.
constexpr int kFillBytes = 32768;
struct FillArgs {
  void* dw[kMaxK];
  int64_t bytes;                        // of a language's gradient
  int64_t units, from, own;             // kFillBytes in a gradient; the first here; CTAs ahead of them
};
__device__ __forceinline__ void fill(const FillArgs& a) {
  const int64_t i = a.from + blockIdx.x - a.own, k = i / a.units, u = i - k * a.units;
  char* p = static_cast<char*>(a.dw[k]);
  const int64_t ahead = (int64_t)(-(uintptr_t)p & 15), whole = a.bytes > ahead ? (a.bytes - ahead) & ~(int64_t)15 : 0;
  if (u == 0) {                         // what lies outside the whole vectors, by 2 bytes
    const int64_t c = threadIdx.x < 8 ? 2 * threadIdx.x : ahead + whole + 2 * (threadIdx.x - 8);
    if (threadIdx.x < 16 && c < (threadIdx.x < 8 ? (ahead < a.bytes ? ahead : a.bytes) : a.bytes))
      *reinterpret_cast<uint16_t*>(p + c) = 0;
  }
#pragma unroll
  for (int j = 0; j < kFillBytes / 16 / kEmbedThreads; ++j) {
    const int64_t c = u * kFillBytes + 16 * (j * kEmbedThreads + threadIdx.x);
    if (c < whole) *reinterpret_cast<uint4*>(p + ahead + c) = make_uint4(0, 0, 0, 0);
  }
}

// A row's (language, token, t): language and token in the upper half, kNoToken where the
// row has none.
struct OrderArgs {
  const void* ids;
  uint64_t* out;
  int64_t T, V;
  int32_t id_bytes, K;
  int64_t rows[kMaxK + 1];
};
__global__ void __launch_bounds__(kSortRun) sort_runs_kernel(const __grid_constant__ OrderArgs a, const __grid_constant__ FillArgs f) {
  grid_wait();
  if (blockIdx.x >= f.own) return fill(f);
  const int tid = threadIdx.x;
  const int64_t t = (int64_t)blockIdx.x * kSortRun + tid;
  uint64_t mine = ~0ull;
  if (t < a.T) {
    int k = 0;
    while (t >= a.rows[k + 1]) ++k;
    const int64_t id = load_id(a.ids, a.id_bytes, t);
    const uint32_t key = id < 0 || id >= a.V ? kNoToken : (uint32_t)(k * a.V + id);
    mine = (uint64_t)key << 32 | (uint32_t)t;
  }
  __shared__ uint64_t room[kSortRun];
#pragma unroll 1
  for (int size = 2; size <= kSortRun; size *= 2) {
#pragma unroll 1
    for (int step = size / 2; step > 0; step /= 2) {
      uint64_t other;
      if (step >= 32) {
        __syncthreads();
        room[tid] = mine;
        __syncthreads();
        other = room[tid ^ step];
      } else {
        other = __shfl_xor_sync(0xffffffffu, mine, step);
      }
      const bool low = ((tid & step) == 0) == ((tid & size) == 0);
      mine = (mine < other) == low ? mine : other;
    }
  }
  if (t < a.T) a.out[t] = mine;
}

// The first merge: a CTA for 64 rows of a run of kSortRun, 4 threads a row with 8 runs each.
// The keys alone lie in shared memory: equal ones are in the order of their runs.
struct MergeArgs {
  const uint64_t* in;
  uint64_t* out;
  int64_t T, run;
};
constexpr int kMergeRows = kEmbedThreads / 4;
__global__ void __launch_bounds__(kEmbedThreads) merge_keys_kernel(const __grid_constant__ MergeArgs a, const __grid_constant__ FillArgs f) {
  grid_wait();
  if (blockIdx.x >= f.own) return fill(f);
  // (run r's place i lies at i ^ r: the same place of other runs is in other banks)
  __shared__ uint32_t keys[kMerge][kSortRun];
  const int tid = threadIdx.x;
  const int64_t own = (int64_t)blockIdx.x * kMergeRows / kSortRun, first = own / kMerge * kMerge * kSortRun;
#pragma unroll
  for (int j = 0; j < kMerge; ++j) {
    const int64_t i = first + j * kSortRun + tid;
    keys[j][tid ^ j] = i < a.T ? (uint32_t)(a.in[i] >> 32) : kNoToken;
  }
  const int64_t i = (int64_t)blockIdx.x * kMergeRows + tid / 4;
  const uint64_t mine = i < a.T ? a.in[i] : ~0ull;
  const uint32_t key = (uint32_t)(mine >> 32);
  const int me = (int)(own % kMerge);
  __syncthreads();
  // places of each run that come before this row
  int before[kMerge / 4] = {};
#pragma unroll
  for (int step = kSortRun / 2; step > 0; step /= 2) {
#pragma unroll
    for (int j = 0; j < kMerge / 4; ++j) {
      const int r = 4 * j + (tid & 3);
      const uint32_t there = keys[r][(before[j] + step - 1) ^ r];
      if (there < key || (there == key && r < me)) before[j] += step;
    }
  }
  int place = 0;
#pragma unroll
  for (int j = 0; j < kMerge / 4; ++j) {
    const int r = 4 * j + (tid & 3);
    if (r == me) continue;
    const uint32_t there = keys[r][before[j] ^ r];          // (all but one have been looked at)
    place += before[j] + (there < key || (there == key && r < me) ? 1 : 0);
  }
  place += __shfl_xor_sync(0xffffffffu, place, 1);
  place += __shfl_xor_sync(0xffffffffu, place, 2);
  if (i < a.T && (tid & 3) == 0) a.out[first + (i - own * kSortRun) + place] = mine;
}

// A later merge: runs of `run` places in groups of kMerge, 8 threads a row with a run each in
// turn.
constexpr int kMergeLanes = 8;
__global__ void __launch_bounds__(kEmbedThreads) merge_runs_kernel(const __grid_constant__ MergeArgs a, const __grid_constant__ FillArgs f) {
  grid_wait();
  if (blockIdx.x >= f.own) return fill(f);
  const int64_t i = ((int64_t)blockIdx.x * kEmbedThreads + threadIdx.x) / kMergeLanes;
  const bool live = i < a.T;
  const uint64_t mine = live ? a.in[i] : 0;
  const int64_t own = i / a.run, group = own / kMerge * kMerge;
  int64_t place = 0;
  for (int j = threadIdx.x % kMergeLanes; j < kMerge; j += kMergeLanes) {
    const int64_t from = (group + j) * a.run;
    if (!live || group + j == own || from >= a.T) continue;
    int64_t lo = 0, hi = a.T - from < a.run ? a.T - from : a.run;      // how many are less than mine
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (a.in[from + mid] < mine) lo = mid + 1;
      else hi = mid;
    }
    place += lo;
  }
#pragma unroll
  for (int w = kMergeLanes / 2; w > 0; w /= 2) place += __shfl_xor_sync(0xffffffffu, place, w);
  if (live && threadIdx.x % kMergeLanes == 0) a.out[group * a.run + (i - own * a.run) + place] = mine;
}

// ---- sums ------------------------------------------------------------------

struct SumArgs {
  const uint64_t* order;
  const void* dy;
  float* part;                          // [piece][2][columns]
  void* dw[kMaxK];
  int64_t ld, T, V, D, ld_part, pieces;
  float scale;
  int32_t accumulate, piece;            // places of a warp, 8 to 32
  uint32_t blocks;                      // of kColumns columns
};

__device__ __forceinline__ uint32_t key_at(const SumArgs& a, int64_t i) {
  return i < 0 || i >= a.T ? kNoToken : (uint32_t)(a.order[i] >> 32);
}

// A lane's 8 columns of a row from c0 on: side by side where rows start on 16 bytes, else 32
// apart; 0 beyond the last column.
template <class E, bool VEC>
struct Eight {
  uint4 v[sizeof(E) / 2];
  __device__ __forceinline__ void load(const E* row, int64_t c0, int lane, int64_t D) {
    const int64_t c = c0 + 8 * lane;
#pragma unroll
    for (int j = 0; j < (int)sizeof(E) / 2; ++j) {
      v[j] = make_uint4(0, 0, 0, 0);
      if (c + j * kVec<E> < D) v[j] = reinterpret_cast<const uint4*>(row + c)[j];
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < (int)sizeof(E) / 2; ++j) {
      float y[kVec<E>];
      unpack(v[j], y);
#pragma unroll
      for (int e = 0; e < kVec<E>; ++e) x[j * kVec<E> + e] = y[e];
    }
  }
  static __device__ __forceinline__ void store(E* row, int64_t c0, int lane, int64_t D, const float (&x)[8]) {
    const int64_t c = c0 + 8 * lane;
#pragma unroll
    for (int j = 0; j < (int)sizeof(E) / 2; ++j) {
      float y[kVec<E>];
#pragma unroll
      for (int e = 0; e < kVec<E>; ++e) y[e] = x[j * kVec<E> + e];
      if (c + j * kVec<E> < D) reinterpret_cast<uint4*>(row + c)[j] = repack(y);
    }
  }
};
template <class E>
struct Eight<E, false> {
  E v[8];
  __device__ __forceinline__ void load(const E* row, int64_t c0, int lane, int64_t D) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c0 + lane + 32 * j < D ? row[c0 + lane + 32 * j] : narrow<E>(0.0f);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = widen(v[j]);
  }
  static __device__ __forceinline__ void store(E* row, int64_t c0, int lane, int64_t D, const float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c0 + lane + 32 * j < D) row[c0 + lane + 32 * j] = narrow<E>(x[j]);
  }
};
// Rows looked up that do not all start on 16 bytes: a warp for 256 columns of one.
template <class E>
__global__ void __launch_bounds__(kEmbedThreads) embed_odd_kernel(const __grid_constant__ LookupArgs a) {
  grid_wait();
  const int lane = threadIdx.x & 31;
  const int64_t n = a.T * a.per;
  for (int64_t i = (int64_t)blockIdx.x * (kEmbedThreads / 32) + (threadIdx.x >> 5); i < n;
       i += (int64_t)gridDim.x * (kEmbedThreads / 32)) {
    const int64_t t = n < (1ll << 32) ? (uint32_t)i / a.per : i / a.per, c0 = (i - t * a.per) * kColumns;
    const int64_t id = load_id(a.ids, a.id_bytes, t);
    float x[8] = {};
    if (id >= 0 && id < a.V) {
      Eight<E, false> v;
      v.load(static_cast<const E*>(a.table) + id * a.ld, c0, lane, a.D);
      v.get(x);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= a.scale;
    Eight<E, false>::store(static_cast<E*>(a.y) + t * a.ld_y, c0, lane, a.D, x);
  }
}
template <class E>
const void* embed_fn(bool vec, bool ahead) {
  return !vec ? (const void*)embed_odd_kernel<E> : ahead ? (const void*)embed_kernel<E, 4> : (const void*)embed_kernel<E, 1>;
}

using Part8 = Eight<float, true>;       // (a lane's 8 columns side by side, whichever they are)

template <class W>
__device__ __forceinline__ W* place_of(const SumArgs& a, uint32_t key) {
  const uint32_t k = key / (uint32_t)a.V, v = key % (uint32_t)a.V;
  return static_cast<W*>(a.dw[k]) + (int64_t)v * a.D;
}
// A finished sum to its place, which held `old`.
template <class W, bool VEC>
__device__ __forceinline__ void finish(const SumArgs& a, W* row, int64_t c0, int lane, const float (&sum)[8], const Eight<W, VEC>& old) {
  float x[8];
  if (a.accumulate) {
    old.get(x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = fmaf(sum[j], a.scale, x[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = sum[j] * a.scale;
  }
  Eight<W, VEC>::store(row, c0, lane, a.D, x);
}
__device__ __forceinline__ float* part_row(const SumArgs& a, int64_t piece, int which, int64_t c0) {
  return a.part + (piece * 2 + which) * a.ld_part + c0;
}

// A warp's piece: places a.piece * piece and on, 256 columns from c0.  What begins before the
// piece goes to its first part, what goes on behind it to its second.  kRowsAhead rows, and
// the places that they are added to, are on their way at once.
// (8 CTAs an SM leave 64 registers: of bf16 sums by vectors 28 bytes a thread go to memory.)
constexpr int kSumThreads = 128;
constexpr int kRowsAhead = 4;
template <class E, class W, bool VEC>
__global__ void __launch_bounds__(kSumThreads, sizeof(E) + sizeof(W) == 4 && VEC ? 8 : 5) sum_pieces_kernel(const __grid_constant__ SumArgs a) {
  grid_wait();
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * (kSumThreads / 32) + (threadIdx.x >> 5);
  const int64_t piece = unit / a.blocks, c0 = (unit - piece * a.blocks) * kColumns;
  if (piece >= a.pieces) return;
  const int64_t at = piece * a.piece;
  const bool in = lane < a.piece;
  const uint64_t mine = in && at + lane < a.T ? a.order[at + lane] : ~0ull;
  const uint32_t before = key_at(a, at - 1), behind = key_at(a, at + a.piece);
  const uint32_t key = (uint32_t)(mine >> 32), row = (uint32_t)mine;
  const uint32_t beside = __shfl_down_sync(0xffffffffu, key, 1), next = lane == a.piece - 1 ? behind : beside;
  const int n = __popc(__ballot_sync(0xffffffffu, key != kNoToken));
  const uint32_t ends = __ballot_sync(0xffffffffu, key != kNoToken && key != next);
  const bool first = n > 0 && __shfl_sync(0xffffffffu, key, 0) == before;      // the sum began before the piece
  const uint32_t whole = first ? ends & (ends - 1) : ends;      // ends of the sums that began here
  // each lane's own row and the place that it is added to
  const uint64_t from = (uint64_t)(static_cast<const E*>(a.dy) + (int64_t)row * a.ld);
  const uint64_t place = key == kNoToken ? 0 : (uint64_t)place_of<W>(a, key);
  float sum[8] = {};
  for (int i0 = 0; i0 < n; i0 += kRowsAhead) {
    Eight<E, VEC> dy[kRowsAhead];
    Eight<W, VEC> old[kRowsAhead];
#pragma unroll
    for (int j = 0; j < kRowsAhead; ++j)
      if (i0 + j < n) dy[j].load(reinterpret_cast<const E*>(__shfl_sync(0xffffffffu, from, i0 + j)), c0, lane, a.D);
    if (a.accumulate) {
#pragma unroll
      for (int j = 0; j < kRowsAhead; ++j)
        if (whole >> (i0 + j) & 1)
          old[j].load(reinterpret_cast<const W*>(__shfl_sync(0xffffffffu, place, i0 + j)), c0, lane, a.D);
    }
#pragma unroll
    for (int j = 0; j < kRowsAhead; ++j) {
      if (i0 + j >= n) break;
      float x[8];
      dy[j].get(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += x[e];
      if (whole >> (i0 + j) & 1) {
        finish<W, VEC>(a, reinterpret_cast<W*>(__shfl_sync(0xffffffffu, place, i0 + j)), c0, lane, sum, old[j]);
      } else if (ends >> (i0 + j) & 1) {
        Part8::store(part_row(a, piece, 0, c0), 0, lane, kColumns, sum);
      } else if (i0 + j == n - 1) {     // goes on
        Part8::store(part_row(a, piece, first && ends == 0 ? 0 : 1, c0), 0, lane, kColumns, sum);
      } else {
        continue;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    }
  }
}

// Parts from .. to - 1 of pieces in which a sum goes on, added to `sum`.
__device__ __forceinline__ void add_parts(const SumArgs& a, int64_t from, int64_t to, int64_t c0, int lane, float (&sum)[8]) {
  constexpr int kAhead = 4;
  for (int64_t p = from; p < to; p += kAhead) {
    Part8 v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (p + j < to) v[j].load(part_row(a, p + j, 0, c0), 0, lane, kColumns);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (p + j >= to) break;
      float x[8];
      v[j].get(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += x[e];
    }
  }
}

// The sums of more than one piece, by the warp of the piece in which they begin; by all warps
// of its CTA where they go on for more than 31 pieces.
template <class W, bool VEC>
__global__ void __launch_bounds__(kEmbedThreads) join_pieces_kernel(const __grid_constant__ SumArgs a) {
  grid_wait();
  constexpr int kWarpsHere = kEmbedThreads / 32;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int64_t piece = (int64_t)blockIdx.x * kWarpsHere + wid, c0 = (int64_t)blockIdx.y * kColumns;
  __shared__ int64_t long_piece;
  __shared__ float room[kWarpsHere][kColumns];
  if (threadIdx.x == 0) long_piece = -1;
  __syncthreads();
  // the keys of this piece's last place and of the first ones of those behind it
  const int64_t start = (piece + lane) * a.piece;
  const uint32_t ahead = key_at(a, start), tail = key_at(a, (piece + 1) * a.piece - 1), prior = key_at(a, piece * a.piece - 1);
  const uint32_t head = __shfl_sync(0xffffffffu, ahead, 0);
  const bool begins = piece < a.pieces && tail != kNoToken && !(head == tail && prior == tail);
  const uint32_t same = __ballot_sync(0xffffffffu, lane > 0 && ahead == tail) >> 1;
  const int on = __ffs(~same) - 1;      // pieces behind this one that hold the token, at most 31
  W* to = begins && on > 0 ? place_of<W>(a, tail) : nullptr;
  if (to && on < 31) {
    Eight<W, VEC> old;
    if (a.accumulate) old.load(to, c0, lane, a.D);
    float sum[8];
    Part8 v;
    v.load(part_row(a, piece, 1, c0), 0, lane, kColumns);
    v.get(sum);
    add_parts(a, piece + 1, piece + 1 + on, c0, lane, sum);
    finish<W, VEC>(a, to, c0, lane, sum, old);
  }
  if (to && on >= 31 && lane == 0) long_piece = piece;   // at most one of 8 neighbours
  __syncthreads();
  const int64_t from = long_piece;
  if (from < 0) return;
  const uint32_t key = key_at(a, (from + 1) * a.piece - 1);
  int64_t n = 0;
  for (;;) {
    const int64_t p = from + 1 + n + threadIdx.x;
    const int c = __syncthreads_count(p < a.pieces && key_at(a, p * a.piece) == key);
    n += c;
    if (c < kEmbedThreads) break;
  }
  const int64_t each = (n + kWarpsHere - 1) / kWarpsHere, lo = from + 1 + wid * each, end = from + 1 + n;
  float sum[8] = {};
  if (wid == 0) {
    Part8 v;
    v.load(part_row(a, from, 1, c0), 0, lane, kColumns);
    v.get(sum);
  }
  add_parts(a, lo, lo + each < end ? lo + each : end, c0, lane, sum);
#pragma unroll
  for (int j = 0; j < 8; ++j) room[wid][lane + 32 * j] = sum[j];
  __syncthreads();
  if (wid != 0) return;
  for (int w = 1; w < kWarpsHere; ++w)
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += room[w][lane + 32 * j];
  W* row = place_of<W>(a, key);
  Eight<W, VEC> old;
  if (a.accumulate) old.load(row, c0, lane, a.D);
  finish<W, VEC>(a, row, c0, lane, sum, old);
}

int64_t up_by(int64_t n, int64_t by) { return (n + by - 1) / by; }
bool matrix_ok(const void* p, int32_t dtype, int64_t rows, int64_t cols, int64_t ld) {
  return rows == 0 || (aligned_at(p, float_bytes(dtype)) && ld >= cols && ld <= ((int64_t)1 << 38));
}
bool on_vectors(const void* p, int32_t dtype, int64_t cols, int64_t ld) {
  const uintptr_t e = float_bytes(dtype);
  return (((uintptr_t)p | (uintptr_t)(cols * e) | (uintptr_t)(ld * e)) & 15) == 0;
}
bool embed_sizes_ok(int64_t T, int64_t V, int64_t D, double scale) {
  return T >= 0 && T <= ((int64_t)1 << 31) - 1024 && V >= 1 && V <= ((int64_t)1 << 28) - 1 && D >= 1 &&
         D <= ((int64_t)1 << 23) && std::isfinite((float)scale);
}

// Places of a warp's piece: as many as leave 2432 warps (16 for each of 152 SMs), 8 to 32.
// 600 rows of 768 bf16 in 4 languages, added, take 12, 14 and 18 us by pieces of 8, 16 and 32;
// 8192 of 2048 23, 21 and 22; 65536 of 768 79, 72 and 71.
int piece_of(int64_t T, int64_t blocks) {
  int piece = 32;
  while (piece > 8 && up_by(T, piece) * blocks < 2432) piece /= 2;
  return piece;
}
struct EmbedRoom {
  size_t order[2], part, total;
  int64_t pieces, blocks;
  int piece;
};
EmbedRoom embed_room(int64_t T, int64_t D) {
  EmbedRoom r;
  r.blocks = up_by(D, kColumns);
  r.piece = piece_of(T, r.blocks);
  r.pieces = up_by(T, r.piece);
  r.order[0] = 0;
  r.order[1] = align256((size_t)T * 8);
  r.part = r.order[1] + (T > kSortRun ? align256((size_t)T * 8) : 0);
  r.total = r.part + align256((size_t)r.pieces * 2 * (size_t)r.blocks * kColumns * 4);
  return r;
}

template <class E, class W>
const void* sum_fn(bool vec) {
  return vec ? (const void*)sum_pieces_kernel<E, W, true> : (const void*)sum_pieces_kernel<E, W, false>;
}

}  // namespace
}  // namespace bkmoo

using namespace bkmoo;

extern "C" int bkmoo_embedding_forward(const void* table, int64_t ld_table, int32_t dtype, int64_t V,
                                       int64_t D, const void* ids, int32_t id_bytes, int64_t T,
                                       double scale, void* y, int64_t ldy, void* stream) {
  if (!is_float(dtype) || !is_id(id_bytes) || !embed_sizes_ok(T, V, D, scale) ||
      !matrix_ok(table, dtype, V, D, ld_table))
    return BKMOO_ERR_INVALID;
  if (T == 0) return BKMOO_OK;
  if (!matrix_ok(y, dtype, T, D, ldy) || !aligned_at(ids, id_bytes)) return BKMOO_ERR_INVALID;
  const bool vec = on_vectors(table, dtype, D, ld_table) && on_vectors(y, dtype, D, ldy);
  const int64_t per = vec ? D * (int64_t)float_bytes(dtype) / 16 : up_by(D, kColumns);
  LookupArgs a = {table, ids, y, ld_table, ldy, T, V, id_bytes, (uint32_t)D, (uint32_t)per, (float)scale};
  const bool ahead = vec && T * per > 152 * 2048;
  const void* fn = dtype == BKMOO_F32 ? embed_fn<float>(vec, ahead) : embed_fn<__nv_bfloat16>(vec, ahead);
  const int64_t ctas = up_by(T * per, vec ? kEmbedThreads * (ahead ? 4 : 1) : kEmbedThreads / 32), most = 1 << 20;
  void* list[] = {&a};
  return launch_behind(fn, dim3((unsigned)(ctas < most ? ctas : most)), dim3(kEmbedThreads), list, 0,
                       static_cast<cudaStream_t>(stream), true) == cudaSuccess
             ? BKMOO_OK
             : BKMOO_ERR_CUDA;
}

extern "C" int bkmoo_embedding_backward_workspace_size(int64_t T, int64_t D, size_t* bytes) {
  if (!bytes || !embed_sizes_ok(T, 1, D, 1.0)) return BKMOO_ERR_INVALID;
  *bytes = embed_room(T, D).total;
  return BKMOO_OK;
}

extern "C" int bkmoo_embedding_backward(const void* dy, int64_t ld_dy, int32_t dtype, const void* ids,
                                        int32_t id_bytes, int64_t T, int64_t V, int64_t D, double scale,
                                        int32_t K, const int64_t* rows, void* const* dw,
                                        int32_t dw_dtype, int32_t accumulate, void* ws, size_t ws_bytes,
                                        void* stream) {
  if (!is_float(dtype) || !is_float(dw_dtype) || !is_id(id_bytes) || !embed_sizes_ok(T, V, D, scale) ||
      !languages_ok(rows, K, T) || !dw || !size_ok(V, D) || !matrix_ok(dy, dtype, T, D, ld_dy) ||
      (T > 0 && (!aligned_at(ids, id_bytes) || !aligned_at(ws, 256))))
    return BKMOO_ERR_INVALID;
  bool vec = on_vectors(dy, dtype, D, ld_dy);
  for (int k = 0; k < K; ++k) {
    if (!aligned_at(dw[k], float_bytes(dw_dtype))) return BKMOO_ERR_INVALID;
    vec = vec && on_vectors(dw[k], dw_dtype, D, D);
  }
  if (!apart(dw, K, (size_t)(V * D) * float_bytes(dw_dtype))) return BKMOO_ERR_INVALID;
  const EmbedRoom room = embed_room(T, D);
  const int64_t ctas = up_by(room.pieces * room.blocks, kSumThreads / 32);
  const size_t grad_bytes = (size_t)(V * D) * float_bytes(dw_dtype);
  int64_t levels = 1;                   // kernels of the order
  for (int64_t run = kSortRun; run < T; run *= kMerge) ++levels;
  FillArgs f = {};
  f.bytes = (int64_t)grad_bytes;
  f.units = up_by(f.bytes, kFillBytes);
  for (int k = 0; k < K; ++k) f.dw[k] = dw[k];
  const int64_t fills = accumulate ? 0 : K * f.units;
  if (ctas > 0x7fffffffll || fills + up_by(T, kMergeRows) + up_by(T * kMergeLanes, kEmbedThreads) > 0x7fffffffll)
    return BKMOO_ERR_INVALID;
  if (T > 0 && ws_bytes < room.total) return BKMOO_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (T == 0) {
    for (int k = 0; k < K && !accumulate; ++k)
      if (cudaMemsetAsync(dw[k], 0, grad_bytes, s) != cudaSuccess) return BKMOO_ERR_CUDA;
    return BKMOO_OK;
  }
  char* base = static_cast<char*>(ws);
  uint64_t *order = reinterpret_cast<uint64_t*>(base + room.order[0]), *other = reinterpret_cast<uint64_t*>(base + room.order[1]);
  // the order, and a part of the zeros with each of its kernels
  cudaError_t e = cudaSuccess;
  int64_t run = kSortRun;
  for (int64_t level = 0; level < levels && e == cudaSuccess; ++level) {
    f.from = fills * level / levels;
    f.own = level == 0 ? up_by(T, kSortRun) : level == 1 ? up_by(T, kMergeRows) : up_by(T * kMergeLanes, kEmbedThreads);
    const dim3 grid((unsigned)(f.own + fills * (level + 1) / levels - f.from));
    if (level == 0) {
      OrderArgs o = {ids, order, T, V, id_bytes, K, {}};
      for (int k = 0; k <= K; ++k) o.rows[k] = rows[k];
      void* list[] = {&o, &f};
      e = launch_behind((const void*)sort_runs_kernel, grid, dim3(kSortRun), list, 0, s, true);
      continue;
    }
    MergeArgs m = {order, other, T, run};
    void* list[] = {&m, &f};
    e = launch_behind(level == 1 ? (const void*)merge_keys_kernel : (const void*)merge_runs_kernel, grid, dim3(kEmbedThreads), list, 0, s,
                      true);
    run *= kMerge;
    uint64_t* t = order;
    order = other;
    other = t;
  }
  if (e != cudaSuccess) return BKMOO_ERR_CUDA;
  SumArgs a = {order, dy, reinterpret_cast<float*>(base + room.part), {}, ld_dy, T, V, D, room.blocks * kColumns, room.pieces,
               (float)scale, accumulate, room.piece, (uint32_t)room.blocks};
  for (int k = 0; k < K; ++k) a.dw[k] = dw[k];
  void* list[] = {&a};
  const bool wide = dw_dtype == BKMOO_F32;
  const void* fn = dtype == BKMOO_F32 ? wide ? sum_fn<float, float>(vec) : sum_fn<float, __nv_bfloat16>(vec)
                   : wide ? sum_fn<__nv_bfloat16, float>(vec)
                          : sum_fn<__nv_bfloat16, __nv_bfloat16>(vec);
  e = launch_behind(fn, dim3((unsigned)ctas), dim3(kSumThreads), list, 0, s, true);
  if (e == cudaSuccess && room.pieces > 1) {
    fn = wide ? vec ? (const void*)join_pieces_kernel<float, true> : (const void*)join_pieces_kernel<float, false>
         : vec ? (const void*)join_pieces_kernel<__nv_bfloat16, true>
               : (const void*)join_pieces_kernel<__nv_bfloat16, false>;
    e = launch_behind(fn, dim3((unsigned)up_by(room.pieces - 1, kEmbedThreads / 32), a.blocks), dim3(kEmbedThreads), list, 0, s, true);
  }
  return e == cudaSuccess ? BKMOO_OK : BKMOO_ERR_CUDA;
}
