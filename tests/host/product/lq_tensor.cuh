// The wrappers of csrc/lq_tensor.cuh that products use, as the model of product_roles.cpp has them.
#pragma once
#include <cuda.h>
#include <stdint.h>

#include "cuda_threads.h"

namespace lq {

uint32_t shared_addr(const void *p);          // the CTA's number in its cluster in the upper eight bits
inline bool elect_one() { return threadIdx.x % 32 == 0; }

void bar_init(uint32_t bar, int count);
void bar_arrive(uint32_t bar);
void bar_expect(uint32_t bar, uint32_t bytes);
bool bar_try(uint32_t bar, uint32_t parity);
inline void fence_async_shared() { yield(); }
void tensor_g2s(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar);
void tensor_s2g(const CUtensorMap *map, uint32_t src, int x, int y, int z);
void copies_commit();
void wait_for_copies(int but);
template <int N> void copies_read() { wait_for_copies(N); }
inline void copies_done() { wait_for_copies(0); }
inline void tensor_map_prefetch(const CUtensorMap *) {}

void tmem_alloc(uint32_t result_in_shared, int columns);
void tmem_free(uint32_t tmem, int columns);
inline void pair_tmem_alloc(uint32_t result, int columns) { tmem_alloc(result, columns); }
inline void pair_tmem_free(uint32_t tmem, int columns) { tmem_free(tmem, columns); }
inline void tmem_fence_before() {}
inline void tmem_fence_after() {}
void tmem_load16(uint32_t at, uint32_t (&r)[16]);
inline void tmem_wait_loads(uint32_t (&)[16]) {}

struct Operand {                              // (the model goes by the address alone)
  uint32_t at;
  Operand operator+(uint32_t bytes) const { return {at + bytes}; }
};
inline Operand operand(uint32_t addr, uint32_t, uint32_t) { return {addr}; }
constexpr uint32_t mma_e4m3(int m, int n) { return (uint32_t)m << 16 | n; }
void mma8_ss(uint32_t d, Operand a, Operand b, uint32_t what, bool add);
void pair_mma8_ss(uint32_t d, Operand a, Operand b, uint32_t what, bool add);
void mma_commit(uint32_t bar);
void pair_mma_commit(uint32_t bar);

uint32_t cluster_rank();
inline uint32_t shared_of(uint32_t addr, uint32_t rank) { return (addr & 0xFFFFFF) | rank << 24; }
void bar_arrive_cluster(uint32_t bar);
void cluster_arrive();
void cluster_wait();
inline void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
inline void pair_tensor_g2s(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) { tensor_g2s(dst, map, x, y, z, bar); }
void store_cluster(uint32_t addr, float x);

}  // namespace lq
