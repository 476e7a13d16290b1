// Host helpers of the tile kernels' entry points: tensor maps, launches and the
// device word that notes a wait that gave up.
#pragma once

#include "tile_gemm.cuh"

namespace bkmoo {

// A bf16 matrix that the tile kernels read: rows of `ld` elements.
inline bool operand_ok(const void* p, int64_t rows, int64_t cols, int64_t ld) {
  constexpr int64_t kMost = ((int64_t)1 << 31) - 1024;   // coordinates and tiles are 32 bits
  return p && ((uintptr_t)p & 15u) == 0 && rows >= 0 && rows <= kMost && cols >= 1 &&
         cols <= kMost && rows * cols <= ((int64_t)1 << 42) && ld >= cols && ld % 8 == 0 &&
         ld <= ((int64_t)1 << 38);
}
// A language's weight gradient (32 of them at most).
inline bool size_ok(int64_t M, int64_t N) {
  constexpr int64_t kMost = ((int64_t)1 << 31) - 1024;
  return M >= 1 && N >= 1 && M <= kMost && N <= kMost && M * N <= ((int64_t)1 << 37);
}
// Language bounds: 0 = rows[0] <= rows[1] <= ... <= rows[K] = T.
inline bool languages_ok(const int64_t* rows, int32_t K, int64_t T) {
  if (!rows || K < 1 || K > kMaxK || rows[0] != 0 || rows[K] != T) return false;
  for (int k = 0; k < K; ++k)
    if (rows[k + 1] < rows[k]) return false;
  return true;
}
// Widest store that 32-column pieces of every row allow (TileOut).
inline int store_width(const void* p, int64_t ld, int elem) {
  const uintptr_t at = (uintptr_t)p | (uintptr_t)(ld * elem);
  return (at & 31u) == 0 ? 32 : (at & 15u) == 0 ? 16 : (at & 3u) == 0 ? 4 : 0;
}

// Map of a matrix (rows x cols bf16, rows of ld elements) read in boxes of 64
// columns by box_rows rows.
int tile_map(CUtensorMap* m, const void* p, int64_t rows, int64_t cols, int64_t ld, int box_rows);
// SMs of the current device.
int tile_sms(int* sms);
// A tile's shape: CTAs that share it and its columns.
struct TileShape {
  int cg, bn;
};
// rows x cols results (gate: cols of h, of which a tile has bn / 2), `mats` products
// each with `groups` sums of nkt steps.
struct TileSet {
  int64_t rows, cols;
  bool gate;
  const int32_t* nkt;
  int groups, mats;
};
// The shape for one set, or two in turn, and the second's head start (Walk); mode: how
// weight gradients are written (TileMode).
TileShape tile_shape(const TileSet& a, const TileSet* b, int mode, int sms, int32_t* head_start);
// Queues the self-test of a single wait.
int launch_wait_runs_out(int32_t* status, cudaStream_t s);
// Queues a tile kernel over `tiles` tiles.
int tile_launch(const void* fn, TileShape shape, void* args, int64_t tiles, cudaStream_t s);

}  // namespace bkmoo
