// Fifth-generation tensor cores and tensor copies: thin wrappers of the instructions, operand and instruction descriptors.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace lq {

__device__ __forceinline__ uint32_t shared_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// One lane of a converged warp.  (Not `lane == 0`: behind elect the compiler keeps descriptors in uniform registers, and eight matrix
// instructions are issued in 530 clocks next to 24 busy warps instead of in 960.)
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p;
}

// ---- mbarriers ----
__device__ __forceinline__ void bar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// One try, for which the warp may be suspended (for a time of the hardware's choosing).
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done;
}

// Writes of ordinary stores to shared memory become visible to tensor copies and matrix instructions.
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor copy, global -> shared, three coordinates ----
__device__ __forceinline__ void tensor_g2s(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
               "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
               : "memory");
}

// shared -> global: rows and channels beyond the array's end are left out
__device__ __forceinline__ void tensor_s2g(const CUtensorMap *map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// This thread's copies but the last N have read their shared memory / all are done.
template <int N>
__device__ __forceinline__ void copies_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ void tensor_map_prefetch(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// ---- tensor memory ----
__device__ __forceinline__ void tmem_alloc(uint32_t result_in_shared, int columns) {   // one warp
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(result_in_shared), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, int columns) {                // the same warp
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Columns of the lane that belongs to a thread
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(at));
}
// Waits for this thread's loads; the registers are named, so that nothing that uses them can be moved in front of the wait.
__device__ __forceinline__ void tmem_wait_loads(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :: "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
      "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(at)
      : "memory");
}

__device__ __forceinline__ void tmem_store8(uint32_t at, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
               "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(at)
               : "memory");
}
// Sixteen lanes by eight columns, from four 8 x 8 matrices of 16-bit pairs as ldmatrix leaves them: lanes 0 - 7 and 8 - 15 by columns 0 - 3, the
// same by columns 4 - 7
__device__ __forceinline__ void tmem_store_16x8(uint32_t at, const uint32_t (&r)[4]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x2.b32 [%4], {%0, %1, %2, %3};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(at) : "memory");
}

// ---- matrix instructions (bf16 operands, binary32 accumulators) ----
// Shared-memory operand with 128-byte swizzle: rows of 128 bytes, eight rows to a 1024-byte atom.
//  K along the 128 bytes: `group` = bytes from eight rows to the next eight; a K step of 16 is 32 bytes further, `block` is not looked at.
//  M or N along the 128 bytes (64 elements): `group` = bytes from eight K to the next eight, `block` = bytes from 64 elements of M or N to
//  the next 64; a K step of 16 is 2048 bytes further.
// The upper half is a constant of the layout; the lower half is the address in units of 16 bytes and `block`, so that a step through an
// operand is one addition - a single thread issues the matrix instructions, and with descriptors built from scratch it is slower than they are.
struct Operand {
  uint32_t low, high;
  __device__ __forceinline__ Operand operator+(uint32_t bytes) const { return {low + (bytes >> 4), high}; }
};
__device__ __forceinline__ Operand operand(uint32_t addr, uint32_t block, uint32_t group) {
  return {(addr >> 4) | (block >> 4) << 16, (group >> 4) | 1u << 14 | 2u << 29};   // (shared addresses are below 2^18)
}
// Instruction descriptor: binary32 accumulators, bf16 operands; a_mn / b_mn: M (N) is the contiguous direction of A (B).
__host__ __device__ constexpr uint32_t mma_bf16(int m, int n, bool a_mn, bool b_mn) {
  return 1u << 4 | 1u << 7 | 1u << 10 | (a_mn ? 1u : 0u) << 15 | (b_mn ? 1u : 0u) << 16 | (uint32_t)(n / 8) << 17 | (uint32_t)(m / 16) << 24;
}
template <bool ADD>
__device__ __forceinline__ void mma_ss(uint32_t d, Operand a, Operand b, uint32_t what) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.u32 p, %6, 0;\n mov.b64 a, {%1, %2};\n mov.b64 b, {%3, %4};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n}\n" ::"r"(d), "r"(a.low), "r"(a.high), "r"(b.low), "r"(b.high), "r"(what), "n"(ADD)
      : "memory");
}
__device__ __forceinline__ void mma_ss(uint32_t d, Operand a, Operand b, uint32_t what, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.u32 p, %6, 0;\n mov.b64 a, {%1, %2};\n mov.b64 b, {%3, %4};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n}\n" ::"r"(d), "r"(a.low), "r"(a.high), "r"(b.low), "r"(b.high), "r"(what),
      "r"((uint32_t)add)
      : "memory");
}
template <bool ADD>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, Operand b, uint32_t what) {   // A in tensor memory
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 b;\n setp.ne.u32 p, %5, 0;\n mov.b64 b, {%2, %3};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n}\n" ::"r"(d), "r"(a), "r"(b.low), "r"(b.high), "r"(what), "n"(ADD)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, Operand b, uint32_t what, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 b;\n setp.ne.u32 p, %5, 0;\n mov.b64 b, {%2, %3};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n}\n" ::"r"(d), "r"(a), "r"(b.low), "r"(b.high), "r"(what), "r"((uint32_t)add)
      : "memory");
}
// e4m3 operands, both with K along the 128 bytes (a K step of 32 is 32 bytes further), binary32 accumulators.
__host__ __device__ constexpr uint32_t mma_e4m3(int m, int n) { return 1u << 4 | (uint32_t)(n / 8) << 17 | (uint32_t)(m / 16) << 24; }
__device__ __forceinline__ void mma8_ss(uint32_t d, Operand a, Operand b, uint32_t what, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.u32 p, %6, 0;\n mov.b64 a, {%1, %2};\n mov.b64 b, {%3, %4};\n"
      " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %5, p;\n}\n" ::"r"(d), "r"(a.low), "r"(a.high), "r"(b.low), "r"(b.high), "r"(what),
      "r"((uint32_t)add)
      : "memory");
}
// The barrier completes when every matrix instruction that this thread has issued has.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- pairs of CTAs (a cluster of two): one product over both, each with half of the rows of either operand in its shared memory ----
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// The address of the same variable in another CTA of the cluster
__device__ __forceinline__ uint32_t shared_of(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// (Orders tensor memory's reads behind tmem_fence_before, and nothing that is in memory: with .release.cluster it waits for all of the thread's stores, and a
// K block of a product took 1.25 us instead of 0.55.)
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
// All threads of the cluster, whole warps
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
// To this CTA's shared memory, `bar` in either CTA's
__device__ __forceinline__ void pair_tensor_g2s(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
               "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void pair_tmem_alloc(uint32_t result_in_shared, int columns) {   // one warp of either CTA
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(result_in_shared), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void pair_tmem_free(uint32_t tmem, int columns) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
}
__device__ __forceinline__ void pair_mma8_ss(uint32_t d, Operand a, Operand b, uint32_t what, bool add) {   // the first CTA of the pair
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.u32 p, %6, 0;\n mov.b64 a, {%1, %2};\n mov.b64 b, {%3, %4};\n"
      " tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a, b, %5, p;\n}\n" ::"r"(d), "r"(a.low), "r"(a.high), "r"(b.low), "r"(b.high), "r"(what),
      "r"((uint32_t)add)
      : "memory");
}
// The barriers at `bar` in both CTAs complete when every matrix instruction that this thread has issued has.
__device__ __forceinline__ void pair_mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}

// Two binary32 values as bf16, nearest even; `lo` at the lower address.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {   // within 2 steps of 2^-23; results below 2^-126 are 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

}  // namespace lq
