// Rows of an embedding looked up by token and scaled, and the gradient of the embedding
// apart by language (include/bkmoo.h).
//
// Forward: y_t = s W[id_t].  Bound by memory.
//
// Backward: dW_k[v] = s sum of dy_t over language k's rows t with id_t = v.  The rows are
// put in the order of (language, token, t); then each token's rows lie side by side, and
// a warp sums a piece of 32 places for 256 columns in that order.  A sum that lies in one
// piece is written (or added) by its warp; the others leave their parts, which are joined in
// the order of the pieces: no atomics on values, the same result every time.
//
// The order: places of 1024 rows sorted by a CTA (bitonic, in registers and shared memory),
// then runs of sorted rows merged 32 at a time: a row's place in the merged run is its
// place in its own plus, for each other run, how many there come before it, a binary search.
#include <math.h>

#include "tile_host.cuh"
#include "row_ops.cuh"

namespace bkmoo {
namespace {

constexpr int kEmbedThreads = 256;
constexpr int kSortRun = 1024;          // rows that a CTA sorts
constexpr int kMerge = 32;              // runs merged at once
constexpr int kPiece = 32;              // places of a warp
constexpr int kColumns = 256;           // columns of a warp: 8 a lane
constexpr uint32_t kNoToken = 0xffffffffu;

// ---- forward ---------------------------------------------------------------

struct LookupArgs {
  const void *table, *ids;
  void* y;
  int64_t ld, ld_y, T, V;
  int32_t id_bytes;
  uint32_t D, per;                      // columns; threads' pieces of a row
  float scale;
};
// VEC: 16 bytes a thread at a time, else an element.
template <class E, bool VEC>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const LookupArgs a) {
  grid_wait();
  constexpr int N = VEC ? kVec<E> : 1;
  const int64_t n = a.T * a.per;
  for (int64_t i = (int64_t)blockIdx.x * kEmbedThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kEmbedThreads) {
    const int64_t t = n < (1ll << 32) ? (uint32_t)i / a.per : i / a.per;
    const int64_t c = (i - t * a.per) * N;
    const int64_t id = load_id(a.ids, a.id_bytes, t);
    const bool none = id < 0 || id >= a.V;
    const E* from = static_cast<const E*>(a.table) + (none ? 0 : id) * a.ld + c;
    E* to = static_cast<E*>(a.y) + t * a.ld_y + c;
    if (VEC) {
      float x[kVec<E>] = {};
      if (!none) unpack(*reinterpret_cast<const uint4*>(from), x);
#pragma unroll
      for (int j = 0; j < kVec<E>; ++j) x[j] *= a.scale;
      *reinterpret_cast<uint4*>(to) = repack(x);
    } else {
      *to = narrow<E>(none ? 0.0f : widen(*from) * a.scale);
    }
  }
}

// ---- order -----------------------------------------------------------------

// A row's (language, token, t): language and token in the upper half, kNoToken where the
// row has none.
struct OrderArgs {
  const void* ids;
  uint64_t* out;
  int64_t T, V;
  int32_t id_bytes, K;
  int64_t rows[kMaxK + 1];
};
__global__ void __launch_bounds__(kSortRun) sort_runs_kernel(const OrderArgs a) {
  grid_wait();
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

// Runs of `run` sorted places merged in groups of kMerge.
__global__ void __launch_bounds__(kEmbedThreads)
    merge_runs_kernel(const uint64_t* in, uint64_t* out, const int64_t T, const int64_t run) {
  grid_wait();
  const int64_t i = (int64_t)blockIdx.x * kEmbedThreads + threadIdx.x;
  if (i >= T) return;
  const uint64_t mine = in[i];
  const int64_t own = i / run, group = own / kMerge * kMerge;
  int64_t place = group * run + (i - own * run);
#pragma unroll 4
  for (int j = 0; j < kMerge; ++j) {
    const int64_t from = (group + j) * run;
    if (group + j == own || from >= T) continue;
    int64_t lo = 0, hi = T - from < run ? T - from : run;      // how many are less than mine
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (in[from + mid] < mine) lo = mid + 1;
      else hi = mid;
    }
    place += lo;
  }
  out[place] = mine;
}

// ---- sums ------------------------------------------------------------------

struct SumArgs {
  const uint64_t* order;
  const void* dy;
  float* part;                          // [piece][2][columns]
  void* dw[kMaxK];
  int64_t ld, T, V, D, ld_part;
  float scale;
  int32_t accumulate;
};

__device__ __forceinline__ uint32_t key_at(const SumArgs& a, int64_t i) {
  return i < 0 || i >= a.T ? kNoToken : (uint32_t)(a.order[i] >> 32);
}

// A lane's 8 columns: side by side where rows start on 16 bytes, else 32 apart.
template <bool VEC>
__device__ __forceinline__ int64_t column(int64_t c0, int lane, int j) {
  return VEC ? c0 + 8 * lane + j : c0 + lane + 32 * j;
}
template <class E, bool VEC>
__device__ __forceinline__ void load8(const E* row, int64_t c0, int lane, int64_t D, float (&x)[8]) {
  if (VEC) {
    const int64_t c = c0 + 8 * lane;
    const uint4* p = reinterpret_cast<const uint4*>(row + c);
    if (sizeof(E) == 2) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (c < D) v = p[0];
      unpack(v, x);
    } else {
      uint4 v[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
      if (c < D) v[0] = p[0];
      if (c + 4 < D) v[1] = p[1];
      float y[4], z[4];
      unpack(v[0], y);
      unpack(v[1], z);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = y[j], x[j + 4] = z[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t c = column<false>(c0, lane, j);
      x[j] = c < D ? widen(row[c]) : 0.0f;
    }
  }
}
template <class E, bool VEC>
__device__ __forceinline__ void store8(E* row, int64_t c0, int lane, int64_t D, const float (&x)[8]) {
  if (VEC) {
    const int64_t c = c0 + 8 * lane;
    uint4* p = reinterpret_cast<uint4*>(row + c);
    if (sizeof(E) == 2) {
      if (c < D) p[0] = repack(x);
    } else {
      const float y[4] = {x[0], x[1], x[2], x[3]}, z[4] = {x[4], x[5], x[6], x[7]};
      if (c < D) p[0] = repack(y);
      if (c + 4 < D) p[1] = repack(z);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t c = column<false>(c0, lane, j);
      if (c < D) row[c] = narrow<E>(x[j]);
    }
  }
}
// A finished sum to its place.
template <class W, bool VEC>
__device__ __forceinline__ void finish(const SumArgs& a, uint32_t key, int64_t c0, int lane, const float (&sum)[8]) {
  const uint32_t k = key / (uint32_t)a.V, v = key % (uint32_t)a.V;
  W* row = static_cast<W*>(a.dw[k]) + (int64_t)v * a.D;
  float x[8];
  if (a.accumulate) {
    load8<W, VEC>(row, c0, lane, a.D, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = fmaf(sum[j], a.scale, x[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = sum[j] * a.scale;
  }
  store8<W, VEC>(row, c0, lane, a.D, x);
}
__device__ __forceinline__ float* part_row(const SumArgs& a, int64_t piece, int which, int64_t c0) {
  return a.part + (piece * 2 + which) * a.ld_part + c0;
}

// A warp's piece: places kPiece * piece and on, 256 columns from c0.  What begins before the
// piece goes to its first part, what goes on behind it to its second.
template <class E, class W, bool VEC>
__global__ void __launch_bounds__(kEmbedThreads) sum_pieces_kernel(const SumArgs a, const uint32_t blocks, const int64_t pieces) {
  grid_wait();
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * (kEmbedThreads / 32) + (threadIdx.x >> 5);
  const int64_t piece = unit / blocks, c0 = (unit - piece * blocks) * kColumns;
  if (piece >= pieces) return;
  const int64_t at = piece * kPiece;
  const uint64_t mine = at + lane < a.T ? a.order[at + lane] : ~0ull;
  const uint32_t key = (uint32_t)(mine >> 32), row = (uint32_t)mine;
  const uint32_t next = key_at(a, at + lane + 1), before = key_at(a, at - 1);
  const int n = __popc(__ballot_sync(0xffffffffu, key != kNoToken));
  const uint32_t ends = __ballot_sync(0xffffffffu, key != next);
  bool first = __shfl_sync(0xffffffffu, key, 0) == before;      // the sum began before the piece
  float sum[8] = {};
  for (int i = 0; i < n; ++i) {
    float x[8];
    load8<E, VEC>(static_cast<const E*>(a.dy) + (int64_t)__shfl_sync(0xffffffffu, row, i) * a.ld, c0, lane, a.D, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += x[j];
    const bool end = ends >> i & 1;
    if (!end && i + 1 < n) continue;
    if (first || !end)
      store8<float, true>(part_row(a, piece, first ? 0 : 1, c0), 0, lane, kColumns, sum);
    else
      finish<W, VEC>(a, __shfl_sync(0xffffffffu, key, i), c0, lane, sum);
    first = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
  }
}

// The sums of more than one piece: a CTA for each piece in which one begins that goes on,
// its warps each a part of the pieces.
template <class W, bool VEC>
__global__ void __launch_bounds__(kEmbedThreads) join_pieces_kernel(const SumArgs a) {
  grid_wait();
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int64_t piece = blockIdx.x, c0 = (int64_t)blockIdx.y * kColumns, last = piece * kPiece + kPiece - 1;
  const uint32_t key = key_at(a, last);
  if (key == kNoToken || key_at(a, last + 1) != key) return;
  if (key_at(a, piece * kPiece) == key && key_at(a, piece * kPiece - 1) == key) return;   // began before
  // the last place that holds the token
  int64_t lo = last + 1, hi = a.T;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if ((uint32_t)(a.order[mid] >> 32) <= key) lo = mid + 1;
    else hi = mid;
  }
  const int64_t end = (lo - 1) / kPiece, n = end - piece;       // pieces behind this one
  const int64_t each = (n + kEmbedThreads / 32 - 1) / (kEmbedThreads / 32);
  const int64_t from = piece + 1 + wid * each, to = from + each <= end ? from + each : end + 1;
  float sum[8] = {};
  if (wid == 0) load8<float, true>(part_row(a, piece, 1, c0), 0, lane, kColumns, sum);
  for (int64_t p = from; p < to; ++p) {
    float x[8];
    load8<float, true>(part_row(a, p, 0, c0), 0, lane, kColumns, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += x[j];
  }
  // (a lane's 8 columns as load8<., VEC> has them, whatever their places in a part)
  __shared__ float room[kEmbedThreads / 32][kColumns];
#pragma unroll
  for (int j = 0; j < 8; ++j) room[wid][lane + 32 * j] = sum[j];
  __syncthreads();
  if (wid != 0) return;
  for (int w = 1; w < kEmbedThreads / 32; ++w)
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += room[w][lane + 32 * j];
  finish<W, VEC>(a, key, c0, lane, sum);
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

struct EmbedRoom {
  size_t order[2], part, total;
  int64_t pieces, blocks;
};
EmbedRoom embed_room(int64_t T, int64_t D) {
  EmbedRoom r;
  r.pieces = up_by(T, kPiece);
  r.blocks = up_by(D, kColumns);
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
  const int n = vec ? (int)(16 / float_bytes(dtype)) : 1;
  LookupArgs a = {table, ids, y, ld_table, ldy, T, V, id_bytes, (uint32_t)D, (uint32_t)(D / n), (float)scale};
  const void* fn = dtype == BKMOO_F32 ? vec ? (const void*)embed_kernel<float, true> : (const void*)embed_kernel<float, false>
                   : vec ? (const void*)embed_kernel<__nv_bfloat16, true>
                         : (const void*)embed_kernel<__nv_bfloat16, false>;
  const int64_t ctas = up_by(T * a.per, kEmbedThreads), most = 1 << 20;
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
  const EmbedRoom room = embed_room(T, D);
  const int64_t ctas = up_by(room.pieces * room.blocks, kEmbedThreads / 32);
  if (ctas > 0x7fffffffll) return BKMOO_ERR_INVALID;
  if (T > 0 && ws_bytes < room.total) return BKMOO_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (!accumulate)
    for (int k = 0; k < K; ++k)
      if (cudaMemsetAsync(dw[k], 0, (size_t)(V * D) * float_bytes(dw_dtype), s) != cudaSuccess) return BKMOO_ERR_CUDA;
  if (T == 0) return BKMOO_OK;
  char* base = static_cast<char*>(ws);
  uint64_t *order = reinterpret_cast<uint64_t*>(base + room.order[0]), *other = reinterpret_cast<uint64_t*>(base + room.order[1]);
  OrderArgs o = {ids, order, T, V, id_bytes, K, {}};
  for (int k = 0; k <= K; ++k) o.rows[k] = rows[k];
  void* sort_list[] = {&o};
  cudaError_t e = launch_behind((const void*)sort_runs_kernel, dim3((unsigned)up_by(T, kSortRun)), dim3(kSortRun), sort_list, 0, s, true);
  for (int64_t run = kSortRun; run < T && e == cudaSuccess; run *= kMerge) {
    void* list[] = {&order, &other, &T, &run};
    e = launch_behind((const void*)merge_runs_kernel, dim3((unsigned)up_by(T, kEmbedThreads)), dim3(kEmbedThreads), list, 0, s, true);
    uint64_t* t = order;
    order = other;
    other = t;
  }
  if (e != cudaSuccess) return BKMOO_ERR_CUDA;
  SumArgs a = {order, dy, reinterpret_cast<float*>(base + room.part), {}, ld_dy, T, V, D, room.blocks * kColumns, (float)scale, accumulate};
  for (int k = 0; k < K; ++k) a.dw[k] = dw[k];
  uint32_t blocks = (uint32_t)room.blocks;
  int64_t pieces = room.pieces;
  void* sum_list[] = {&a, &blocks, &pieces};
  const bool f = dw_dtype == BKMOO_F32;
  const void* fn = dtype == BKMOO_F32 ? f ? sum_fn<float, float>(vec) : sum_fn<float, __nv_bfloat16>(vec)
                   : f ? sum_fn<__nv_bfloat16, float>(vec)
                       : sum_fn<__nv_bfloat16, __nv_bfloat16>(vec);
  e = launch_behind(fn, dim3((unsigned)ctas), dim3(kEmbedThreads), sum_list, 0, s, true);
  if (e == cudaSuccess && pieces > 1) {
    void* list[] = {&a};
    fn = f ? vec ? (const void*)join_pieces_kernel<float, true> : (const void*)join_pieces_kernel<float, false>
         : vec ? (const void*)join_pieces_kernel<__nv_bfloat16, true>
               : (const void*)join_pieces_kernel<__nv_bfloat16, false>;
    e = launch_behind(fn, dim3((unsigned)(pieces - 1), blocks), dim3(kEmbedThreads), list, 0, s, true);
  }
  return e == cudaSuccess ? BKMOO_OK : BKMOO_ERR_CUDA;
}
