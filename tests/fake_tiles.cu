// Tables of tile kernels that are only names: see fake_tiles_runtime.cpp.
#include <cuda.h>

#include <string>

#include "gate_few.cuh"
#include "tile_host.cuh"

void note(const char* what);

static char tables[4][3][257][7];      // [kind][CTAs][columns][mode]: the kernels' addresses

std::string name_of(const void* fn) {
  const char* p = static_cast<const char*>(fn);
  const char* first = &tables[0][0][0][0];
  if (p < first || p >= first + sizeof(tables)) return "pass";
  const int64_t i = p - first;
  static const char* kinds[] = {"gate", "input", "weight", "both"};
  static const char* modes[] = {"plain", "added", "turned", "sums", "sums-turned", "sums-added",
                                "sums-turned-added"};
  return std::string(kinds[i / (3 * 257 * 7)]) + "-" + std::to_string(i / (257 * 7) % 3) + "x" +
         std::to_string(i / 7 % 257) + "-" + modes[i % 7];
}

namespace bkmoo {
const void* tile_gate_fn(int cg, int bn) { return &tables[kGate][cg][bn][kPlain]; }
const void* tile_weight_fn(int cg, int bn, int mode) { return &tables[kWeight][cg][bn][mode]; }
const void* tile_both_fn(int cg, int bn, int mode) { return &tables[kBoth][cg][bn][mode]; }
cudaError_t launch_gate_few(const FewArgs&, int, cudaStream_t) {
  note("few");
  return cudaSuccess;
}
}  // namespace bkmoo
