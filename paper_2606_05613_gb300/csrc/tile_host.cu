// Host side shared by the entry points on the tile kernels (tile_host.cuh), and
// bkmoo_op_status.
#include "tile_host.cuh"

#include <cmath>
#include <mutex>

namespace bkmoo {
namespace {

constexpr int kMaxDevices = 64;

// BKMOO_OK, or the first error of a tile kernel since it was last read (report_give_up).
__device__ int32_t g_status[2];

struct PerDevice {
  void* status = nullptr;
  int sms = 0;
};
std::mutex g_mu;
PerDevice g_dev[kMaxDevices];

int current_device(int* dev) {
  if (cudaGetDevice(dev) != cudaSuccess || *dev < 0 || *dev >= kMaxDevices) return BKMOO_ERR_CUDA;
  return BKMOO_OK;
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                              const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
// Two waits on an arrival that nothing makes, the second of which finds that the first has
// given up, and its report as the tile kernels make it.
__global__ void wait_runs_out_kernel(int32_t* status, uint64_t limit) {
  __shared__ uint64_t bar;
  __shared__ volatile int abort;
  if (threadIdx.x == 0) {
    bar_init(&bar, 1);
    abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  const bool first = bar_wait<1>(&bar, 0, &abort, limit), second = bar_wait<1>(&bar, 0, &abort);
  __syncthreads();
  if (threadIdx.x == 0 && !first && !second && abort) report_give_up(status);
}

EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}

}  // namespace

int tile_map(CUtensorMap* m, const void* p, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  const EncodeFn fn = encode_fn();
  if (!fn) return BKMOO_ERR_CUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, step[2] = {1, 1};
  const CUresult r =
      fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, step,
         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? BKMOO_OK : BKMOO_ERR_CUDA;
}

int tile_sms(int* sms) {
  int dev = 0;
  const int r = current_device(&dev);
  if (r != BKMOO_OK) return r;
  std::lock_guard<std::mutex> lk(g_mu);
  if (g_dev[dev].sms == 0 &&
      cudaDeviceGetAttribute(&g_dev[dev].sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return BKMOO_ERR_CUDA;
  *sms = g_dev[dev].sms;
  return BKMOO_OK;
}

// Outside stream capture the address is looked up on every call, so that a
// context rebuilt after cudaDeviceReset gets its own; a call made while `s` is
// being captured takes the last one seen on the device.
int tile_status_word(cudaStream_t s, int32_t** word) {
  int dev = 0;
  const int r = current_device(&dev);
  if (r != BKMOO_OK) return r;
  cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
  const bool capturing =
      cudaStreamIsCapturing(s, &cap) != cudaSuccess || cap != cudaStreamCaptureStatusNone;
  if (capturing) (void)cudaGetLastError();
  std::lock_guard<std::mutex> lk(g_mu);
  if (!capturing) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_status) != cudaSuccess || !p) return BKMOO_ERR_CUDA;
    g_dev[dev].status = p;
  }
  if (!g_dev[dev].status) return BKMOO_ERR_CUDA;   // first call on this device during capture
  *word = static_cast<int32_t*>(g_dev[dev].status);
  return BKMOO_OK;
}

// Time of a tile (us) from sweeps on GB300 (forward 9 to 4000 rows, input gradient 16
// to 4000, weight gradients of 16 to 8192 rows in 1, 4 and 8 languages, widths 256 to
// 12288): a step of the sum where the SMs are full, a tile's way to memory (under the
// next tile's sum if that is longer), and a launch with its first and last tile.  What
// the shapes take, us (64 / 128 / 256 columns / pair of 256): forward 2048 -> 8192, 64
// rows 18.7 / 17.0 / 18.5 / 18.5, 2000 rows 156 / 109 / 94 / 79; 4096 -> 12288, 64 rows
// 42.5 / 42.8 / 37.4 / 48.9; input gradient 768 <- 2048, 1000 rows 17.8 / 18.1 / 26.1 /
// 26.6, 4000 rows 48 / 38 / 36 / 35; weight gradient 2048 x 768, 4 languages of 128 rows
// 8.0 / 6.7 / 7.1 / 9.2, of 2048 37 / 23 / 25 / 25; 8192 x 2048, 8 languages of 64 rows 96
// / 66 / 47 / 70, of 1024 341 / 203 / 179 / 157.
struct TileCost {
  TileShape s;
  double step, out, launch;
};
constexpr TileCost kCosts[4] = {{{1, 64}, 0.165, 0.85, 3.5},
                                {{1, 128}, 0.217, 1.15, 3.7},
                                {{1, 256}, 0.360, 1.70, 4.6},
                                {{2, 256}, 0.320, 2.40, 6.0}};
// fp32 results, whose sums are taken in pieces (a pair of 128 columns was no faster
// than one CTA's anywhere: 8192 x 2048, 16384 rows 444 us, 425).  8192 x 2048, 8 languages
// of 64 rows 133 / 141, of 1024 372 / 269.
constexpr TileCost kExactCosts[2] = {{{1, 64}, 0.190, 1.2, 3.6}, {{1, 128}, 0.237, 2.5, 5.1}};
// Tiles of a set, and the mean and the longest time of one.
struct SetCost {
  int64_t tiles = 0;
  double mean = 0.0, longest = 0.0;
};
SetCost set_cost(const TileSet& s, const TileCost& c) {
  const int64_t m = kTileM * c.s.cg, n = s.gate ? c.s.bn / 2 : c.s.bn;
  SetCost r;
  r.tiles = (s.rows + m - 1) / m * ((s.cols + n - 1) / n) * s.mats * s.groups;
  for (int g = 0; g < s.groups; ++g) {
    const double t = s.nkt[g] * c.step > c.out ? s.nkt[g] * c.step : c.out;
    r.longest = t > r.longest ? t : r.longest;
    r.mean += t / s.groups;
  }
  return r;
}
// Sums taken in pieces (kExactSteps) have shapes of their own.  bf16 gradients that are
// turned take 128 columns at most: a kernel of 256 that wrote such gradients ended in a
// fault of the GPU whose cause was not found, so there is none.
TileShape tile_shape(const TileSet& a, const TileSet* b, int mode, int sms, int32_t* head_start) {
  const bool exact = mode_f32(mode);
  const int shapes = exact || mode == kTurned ? 2 : 4;
  TileShape best = kCosts[0].s;
  double least = 0.0;
  for (int i = 0; i < shapes; ++i) {
    const TileCost& c = exact ? kExactCosts[i] : kCosts[i];
    const int64_t units = sms / c.s.cg;
    const SetCost x = set_cost(a, c);
    const SetCost y = b ? set_cost(*b, c) : SetCost();
    double t = (double)((x.tiles + units - 1) / units) * x.mean;
    int32_t head = 0;
    if (b) {
      // units with a tile of the first set less do the second's meanwhile
      const int64_t more = x.tiles % units, spare = more ? units - more : 0;
      const double fit = x.mean / y.mean;
      head = (int32_t)(fit < 1e6 ? fit : 1e6);
      const double left = (double)y.tiles - (double)spare * head;
      if (left > 0.0) t += std::ceil(left / units) * y.mean;
    }
    if (x.longest > t) t = x.longest;
    if (y.longest > t) t = y.longest;
    t += c.launch;
    if (i == 0 || t < least) {
      least = t;
      best = c.s;
      if (head_start) *head_start = head;
    }
  }
  return best;
}

int tile_launch(const void* fn, TileShape shape, void* args, int64_t tiles, cudaStream_t s) {
  const int cg = shape.cg, smem = tile_smem(cg, shape.bn);
  int sms = 0;
  const int r = tile_sms(&sms);
  if (r != BKMOO_OK) return r;
  // every time: the limit belongs to the context, which may be a new one
  if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
    return BKMOO_ERR_CUDA;
  const int64_t units = sms / cg;
  cudaLaunchConfig_t cfg = {};
  // (the kernel waits at its top for the one ahead of it: launch_behind)
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cg;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)((tiles < units ? tiles : units) * cg));
  cfg.blockDim = dim3(kTileThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  void* list[] = {args};
  return cudaLaunchKernelExC(&cfg, fn, list) == cudaSuccess ? BKMOO_OK : BKMOO_ERR_CUDA;
}

int launch_wait_runs_out(int32_t* status, cudaStream_t s) {
  uint64_t limit = 1000000;
  void* list[] = {&status, &limit};
  return launch_behind((const void*)wait_runs_out_kernel, dim3(1), dim3(32), list, 0, s, false) == cudaSuccess
             ? BKMOO_OK
             : BKMOO_ERR_CUDA;
}

}  // namespace bkmoo

using namespace bkmoo;

extern "C" int bkmoo_op_status(void* stream, int32_t* status) {
  if (!status) return BKMOO_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int32_t* word = nullptr;
  const int r = tile_status_word(s, &word);
  if (r != BKMOO_OK) return r;
  if (cudaMemcpyAsync(status, word, sizeof(int32_t), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaMemsetAsync(word, 0, 2 * sizeof(int32_t), s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess)
    return BKMOO_ERR_CUDA;
  return BKMOO_OK;
}

extern "C" int bkmoo_op_status_copy(void* stream, int32_t* status) {
  if (!status || ((uintptr_t)status & 3u)) return BKMOO_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int32_t* word = nullptr;
  const int r = tile_status_word(s, &word);
  if (r != BKMOO_OK) return r;
  return cudaMemcpyAsync(status, word, sizeof(int32_t), cudaMemcpyDefault, s) == cudaSuccess
             ? BKMOO_OK
             : BKMOO_ERR_CUDA;
}
