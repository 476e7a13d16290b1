// Tensor-core products out of shared memory (tcgen05, accumulators in tensor
// memory), the tiled copies that feed them (TMA) and the waits between the two,
// for one CTA or for a pair of CTAs that share a product.
#pragma once

#include <cuda.h>

#include "bulk_copy.cuh"

namespace bkmoo {

// Waits of the tile kernels end on their own: each is for work of this CTA (or
// pair) in flight, microseconds, and gives up after 2 s (`limit`: of the self-test).
constexpr uint64_t kTileWaitNs = 2000000000ull;

template <int CG>
__device__ __forceinline__ bool bar_try_pair(uint64_t* b, unsigned parity) {
  if (CG == 1) return bar_try(b, parity);
  uint32_t ok;
  asm volatile(
      "{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; "
      "selp.u32 %0, 1, 0, p; }"
      : "=r"(ok)
      : "r"(st_smem(b)), "r"(parity)
      : "memory");
  return ok != 0;
}
// True once the phase is over; false once the CTA has given up (*abort).
template <int CG>
__device__ __forceinline__ bool bar_wait(uint64_t* b, unsigned parity, volatile int* abort,
                                         uint64_t limit = kTileWaitNs) {
  for (int i = 0; i < 64; ++i)
    if (bar_try_pair<CG>(b, parity)) return true;
  const uint64_t t = stream_ns();
  for (;;) {
    for (int i = 0; i < 64; ++i)
      if (bar_try_pair<CG>(b, parity)) return true;
    if (*abort) return false;
    if (stream_ns() - t > limit) {
      *abort = 1;
      return false;
    }
  }
}

// The device's status word and the float behind it (tile_status_word).
__device__ __forceinline__ void report_give_up(int32_t* status) {
  atomicCAS(status, BKMOO_OK, BKMOO_ERR_TIMEOUT);
  status[1] = 0x7fc00000;
}

// Address of `p`'s counterpart in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t peer_smem(const void* p, unsigned rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(st_smem(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void bar_arrive_at(uint32_t addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr)
               : "memory");
}

// A box of a matrix into shared memory; x (elements along a row) and y its
// first column and row, `bar` the shared::cluster address of the barrier that
// counts its bytes.
template <int CG>
__device__ __forceinline__ void tile_load(void* dst, const CUtensorMap* map, int x, int y,
                                          uint32_t bar) {
  if (CG == 1)
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%2, %3}], [%4];" ::"r"(st_smem(dst)),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        ".cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(st_smem(dst)),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

// Shared-memory operand with 128-byte swizzle.  Along k (K-major): rows of 64
// elements, groups of 8 rows 1024 bytes apart.  Across k (MN-major): chunks of
// 64 elements of the row or column index, `chunk` bytes apart, each with its
// rows of k 128 bytes apart (8 of them a group of 1024 bytes).
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t chunk) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)(chunk >> 4) << 16) |
         ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// bf16 operands, fp32 accumulator.
__host__ __device__ constexpr uint32_t product_desc(int m, int n, bool a_across, bool b_across) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((a_across ? 1u : 0u) << 15) |
         ((b_across ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <int CG>
__device__ __forceinline__ void tile_product(uint32_t d, uint64_t a, uint64_t b, uint32_t desc,
                                             bool add) {
  if (CG == 1)
    asm volatile(
        "{ .reg .pred p; setp.ne.u32 p, %4, 0; "
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d),
        "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add)
        : "memory");
  else
    asm volatile(
        "{ .reg .pred p; setp.ne.u32 p, %4, 0; "
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d),
        "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add)
        : "memory");
}
// `bar` (of both CTAs of a pair) is arrived at once the products issued so far
// are done.
template <int CG>
__device__ __forceinline__ void products_arrive(uint64_t* bar) {
  if (CG == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                     st_smem(bar))
                 : "memory");
  else
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 "
        "[%0], %1;" ::"r"(st_smem(bar)),
        "h"((uint16_t)3)
        : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t* slot, int cols) {
  if (CG == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     st_smem(slot)),
                 "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     st_smem(slot)),
                 "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t at, int cols) {
  if (CG == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols));
  else
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols));
}
__device__ __forceinline__ void tc_fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
// 32 columns of the warp's 32 lanes: v[j] = column `at` + j of this thread's lane,
// to be used behind tc_landed(v) only.
__device__ __forceinline__ void tc_load32(uint32_t (&v)[32], uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
      "%12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, "
      "%30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
        "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
        "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
        "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
        "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(at)
      : "memory");
}
// Waits for the loads issued so far, and ties what they loaded to the place
// behind the wait.
__device__ __forceinline__ void tc_landed(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int j = 0; j < 32; ++j) asm volatile("" : "+r"(v[j]));
}

}  // namespace bkmoo
