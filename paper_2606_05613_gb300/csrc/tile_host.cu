// Host side shared by the entry points on the tile kernels (tile_host.cuh), and
// bkmoo_op_status.
#include "tile_host.cuh"

#include <mutex>

namespace bkmoo {
namespace {

constexpr int kMaxDevices = 64;

// BKMOO_OK, or the first error of a tile kernel since it was last read.
__device__ int32_t g_status;

struct PerDevice {
  void* status = nullptr;
  int sms = 0;
  const void* sized[8] = {};    // kernels whose shared-memory limit is raised
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

int tile_launch(const void* fn, int cg, void* args, int64_t tiles, cudaStream_t s) {
  int dev = 0, sms = 0;
  int r = current_device(&dev);
  if (r == BKMOO_OK) r = tile_sms(&sms);
  if (r != BKMOO_OK) return r;
  {
    std::lock_guard<std::mutex> lk(g_mu);
    const void** known = g_dev[dev].sized;
    int i = 0;
    while (i < 8 && known[i] && known[i] != fn) ++i;
    if (i == 8 || !known[i]) {
      if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, tile_smem(cg)) !=
          cudaSuccess)
        return BKMOO_ERR_CUDA;
      if (i < 8) known[i] = fn;
    }
  }
  const int64_t units = sms / cg;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cg;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)((tiles < units ? tiles : units) * cg));
  cfg.blockDim = dim3(kTileThreads);
  cfg.dynamicSmemBytes = tile_smem(cg);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  void* list[] = {args};
  return cudaLaunchKernelExC(&cfg, fn, list) == cudaSuccess ? BKMOO_OK : BKMOO_ERR_CUDA;
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
      cudaMemsetAsync(word, 0, sizeof(int32_t), s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess)
    return BKMOO_ERR_CUDA;
  return BKMOO_OK;
}
