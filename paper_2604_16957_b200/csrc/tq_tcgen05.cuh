// tcgen05, TMEM and tensor-map primitives of libtq (internal), cta_group::1 throughout and never with cluster multicast.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tq_async.cuh"

namespace tq {

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
// one box of a 3-D tensor map into shared memory, completing on an mbarrier
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];\n" ::"l"(map), "r"(x), "r"(y), "r"(z),
               "r"(src)
               : "memory");
}

// ---- work stealing from the launch's own grid: asks for a thread block that has not started; the answer (16 bytes of
// shared memory) completes on the mbarrier.  After a "no" a thread block must not ask again.
__device__ __forceinline__ void steal_ask(uint32_t answer, uint32_t bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];\n" ::"r"(answer), "r"(bar)
               : "memory");
}
// blockIdx.x of the thread block that will not start and is this one's now, or -1
__device__ __forceinline__ int steal_answer(uint32_t answer) {
  uint32_t got, x;
  asm volatile(
      "{\n.reg .b128 v;\n.reg .pred p;\nld.shared.b128 v, [%2];\n"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, v;\nselp.u32 %0, 1, 0, p;\nmov.u32 %1, 0;\n"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, v;\n}\n"
      : "=r"(got), "=r"(x)
      : "r"(answer)
      : "memory");
  return got ? static_cast<int>(x) : -1;
}

// ---- tensor memory: 128 lanes x 512 columns of 32 bits.  Address: column in the low half, lane in the high half.
__device__ __forceinline__ void tmem_alloc(uint32_t smem_dst, uint32_t columns) {  // whole warp
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_dst), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) {  // whole warp
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(addr), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }

#define TQ_R8(a, i) "=r"(a[i]), "=r"(a[i + 1]), "=r"(a[i + 2]), "=r"(a[i + 3]), "=r"(a[i + 4]), "=r"(a[i + 5]), "=r"(a[i + 6]), "=r"(a[i + 7])
#define TQ_W8(a, i) "r"(a[i]), "r"(a[i + 1]), "r"(a[i + 2]), "r"(a[i + 3]), "r"(a[i + 4]), "r"(a[i + 5]), "r"(a[i + 6]), "r"(a[i + 7])
// 32 consecutive columns of the lane's row (the warp's quarter of the lanes is in the address)
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
      "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
      : TQ_R8(r, 0), TQ_R8(r, 8), TQ_R8(r, 16), TQ_R8(r, 24)
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
      "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};\n" ::"r"(addr),
      TQ_W8(r, 0), TQ_W8(r, 8), TQ_W8(r, 16), TQ_W8(r, 24)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};\n" ::"r"(addr),
      TQ_W8(r, 0), TQ_W8(r, 8)
      : "memory");
}

__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"r"(addr), TQ_W8(r, 0) : "memory");
}
// 8 and 16 consecutive columns of the lane's row
__device__ __forceinline__ void tmem_ld8(uint32_t addr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n" : TQ_R8(r, 0) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
      : TQ_R8(r, 0), TQ_R8(r, 8)
      : "r"(addr)
      : "memory");
}
// Rows of an accumulator of 64 rows: the 16 rows of the warp's quarter lie in its first 16 lanes.  Threads 0 .. 15 get
// COLS columns of their row from the address on, threads 16 .. 31 those of the same rows COLS columns further.
template <int COLS>
__device__ __forceinline__ void tmem_ld_halves(uint32_t addr, uint32_t* r) {
  static_assert(COLS == 8 || COLS == 16 || COLS == 32, "");
  if constexpr (COLS == 8) {
    asm volatile("tcgen05.ld.sync.aligned.16x32bx2.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8], 8;\n" : TQ_R8(r, 0) : "r"(addr) : "memory");
  } else if constexpr (COLS == 16) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x32bx2.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16], 16;\n"
        : TQ_R8(r, 0), TQ_R8(r, 8)
        : "r"(addr)
        : "memory");
  } else {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x32bx2.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
        "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32], 32;\n"
        : TQ_R8(r, 0), TQ_R8(r, 8), TQ_R8(r, 16), TQ_R8(r, 24)
        : "r"(addr)
        : "memory");
  }
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm volatile("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float max3(float a, float b, float c) {  // NaN if one of them is
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// ---- descriptors
// Shared-memory operand in 128-byte rows, 128-byte swizzle (what a tensor map with that swizzle writes): groups of 8
// rows are 1024 bytes apart.  K-major (rows along M or N): `lead` is not used.  MN-major (rows along K, 64 elements of
// M or N per row): `lead` is the distance in bytes from one 64-element column of rows to the next.
// Low word (advances by bytes / 16) and high word.
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lead) { return ((addr & 0x3ffff) >> 4) | ((lead >> 4) << 16); }
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);

// kind::f16, fp32 accumulators; `bf16`: type of both operands; `mn_major_b`: rows of B run along K; `negate_a`
__host__ __device__ constexpr uint32_t instr_desc(bool bf16, int m, int n, bool mn_major_b) {
  return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((mn_major_b ? 1u : 0u) << 16) |
         (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}
// kind::i8, both operands K-major: A of unsigned bytes, B of signed ones
__host__ __device__ constexpr uint32_t instr_desc_bytes(int m, int n) {
  return (2u << 4) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}
constexpr uint32_t kNegateA = 1u << 13;
constexpr uint32_t kMnMajorA = 1u << 15;  // rows of A run along K

// One lane of a converged warp, the same one in every call: 1 there, 0 in the others.
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t yes;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(yes));
  return yes;
}
// D (tensor memory) = A B or D + A B, issued by the lane whose `leader` is 1; the operation is asynchronous.  The whole
// warp comes here with the same operands: they live in uniform registers, where the instruction wants them.  (Issued from
// a branch that one lane takes, every operand is moved there first, and the issuing thread, not the tensor cores, sets
// the pace.)  Descriptors come as their constant high word and a low word that is a sum of a register and a constant.
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, bool add) {
  asm volatile(
      "{\n.reg .pred p, q;\n.reg .b64 x, y;\nsetp.ne.u32 p, %5, 0;\nsetp.ne.u32 q, %6, 0;\nmov.b64 x, {%1, %3};\nmov.b64 y, {%2, %3};\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, p;\n}\n" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(static_cast<uint32_t>(add)), "r"(leader)
      : "memory");
}
// the same for bytes (kind::i8, 32-bit whole numbers; see instr_desc_bytes)
__device__ __forceinline__ void mma_ss_bytes(uint32_t leader, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, bool add) {
  asm volatile(
      "{\n.reg .pred p, q;\n.reg .b64 x, y;\nsetp.ne.u32 p, %5, 0;\nsetp.ne.u32 q, %6, 0;\nmov.b64 x, {%1, %3};\nmov.b64 y, {%2, %3};\n"
      "@q tcgen05.mma.cta_group::1.kind::i8 [%0], x, y, %4, p;\n}\n" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(static_cast<uint32_t>(add)), "r"(leader)
      : "memory");
}
// the same with A in tensor memory (two 16-bit elements of K per column)
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d, uint32_t a, uint32_t b_lo, uint32_t hi, uint32_t idesc, bool add) {
  asm volatile(
      "{\n.reg .pred p, q;\n.reg .b64 y;\nsetp.ne.u32 p, %5, 0;\nsetp.ne.u32 q, %6, 0;\nmov.b64 y, {%2, %3};\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n}\n" ::"r"(d),
      "r"(a), "r"(b_lo), "r"(hi), "r"(idesc), "r"(static_cast<uint32_t>(add)), "r"(leader)
      : "memory");
}
// arrives on the mbarrier once every tcgen05.mma that the leader issued before has completed
__device__ __forceinline__ void mma_commit(uint32_t leader, uint32_t bar) {
  asm volatile(
      "{\n.reg .pred q;\nsetp.ne.u32 q, %1, 0;\n"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar),
      "r"(leader)
      : "memory");
}

}  // namespace tq
