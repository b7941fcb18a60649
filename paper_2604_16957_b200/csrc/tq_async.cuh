// Asynchronous-copy primitives of libtq (internal): mbarriers, bulk copies between global and shared memory
// (the TMA unit, never with cluster multicast), and the bounded wait every kernel uses for them.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace tq {

constexpr long long kMaxWaitCycles = 1LL << 22;  // bound of every mbarrier wait: about 2 ms of SM clock

__device__ __forceinline__ void mbar_init(uint32_t bar, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// non-blocking probe of a phase
__device__ __forceinline__ bool mbar_test_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// contiguous global -> shared copy (both 16-byte aligned, size a multiple of 16) completing on an mbarrier
__device__ __forceinline__ void bulk_g2s(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// contiguous shared -> global copy (both 16-byte aligned, size a multiple of 16), tracked by the bulk async-group
__device__ __forceinline__ void bulk_s2g(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;\n" ::: "memory"); }
// wait until at most N committed groups of this thread are still READING their shared-memory source
template <int N>
__device__ __forceinline__ void bulk_wait_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;\n" ::"n"(N) : "memory");
}
// orders this thread's ordinary shared-memory writes before later asynchronous-proxy accesses (bulk stores)
__device__ __forceinline__ void fence_proxy_async_smem() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }

// Bounded wait on an mbarrier phase; false if the copy did not complete within the limit.
static __device__ __noinline__ bool wait_stage_slow(uint32_t bar, uint32_t parity, long long limit) {
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity)) {
    if (clock64() - t0 > limit) return false;
  }
  return true;
}
__device__ __forceinline__ bool wait_stage(uint32_t bar, uint32_t parity, long long limit = kMaxWaitCycles) {
  if (mbar_try_wait(bar, parity)) return true;  // the common case: the copy landed while the warp computed
  return wait_stage_slow(bar, parity, limit);
}

// ---- thread blocks of several roles that wait for one another
// Bounded wait that also gives up when another warp of the thread block has: false, and the block winds down.  (Inline:
// registers cannot be moved between warps, as the kernel does, around a function call.)
constexpr long long kTileWait = 16 * kMaxWaitCycles;  // 35 ms: a wait may span some other role's work on a few tiles
constexpr long long kBlockWait = 1LL << 34;           // 9 s: a wait for the next piece of work may span a whole sequence
__device__ __forceinline__ bool wait_slow(uint32_t bar, uint32_t parity, volatile int* stop, long long limit) {
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity)) {
    if (*stop) return false;
    if (clock64() - t0 > limit) {
      *stop = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool wait_on(uint32_t bar, uint32_t parity, volatile int* stop, long long limit) {
  if (mbar_try_wait(bar, parity)) return true;
  return wait_slow(bar, parity, stop, limit);
}
__device__ __forceinline__ bool wait_stage_inline(uint32_t bar, uint32_t parity, long long limit) {
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity))
    if (clock64() - t0 > limit) return false;
  return true;
}
// the same for a whole warp: all its lanes go on, or none
__device__ __forceinline__ bool warp_wait_on(uint32_t bar, uint32_t parity, volatile int* stop, long long limit) {
  return __all_sync(0xffffffffu, wait_on(bar, parity, stop, limit));
}

}  // namespace tq
