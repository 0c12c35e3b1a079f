// The wrappers of csrc/lq_tensor.cuh, as the model of scan_roles.cpp has them.
#pragma once
#include <cuda.h>
#include <stdint.h>

#include "cuda_on_host.h"

namespace lq {

uint32_t shared_addr(const void *p);
inline bool elect_one() { return true; }

void bar_init(uint32_t bar, int count);
void bar_arrive(uint32_t bar);
void bar_expect(uint32_t bar, uint32_t bytes);
bool bar_try(uint32_t bar, uint32_t parity);
inline void fence_async_shared() { yield(); }
void tensor_g2s(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar);
inline void tensor_map_prefetch(const CUtensorMap *) {}

void tmem_alloc(uint32_t result_in_shared, int columns);
void tmem_free(uint32_t tmem, int columns);
inline void tmem_fence_before() {}
inline void tmem_fence_after() {}
inline void tmem_wait_stores() {}
void tmem_load16(uint32_t at, uint32_t (&r)[16]);
inline void tmem_wait_loads(uint32_t (&)[16]) {}
void tmem_store(uint32_t at, int columns);
inline void tmem_store16(uint32_t at, const uint32_t (&)[16]) { tmem_store(at, 16); }
inline void tmem_store8(uint32_t at, const uint32_t (&)[8]) { tmem_store(at, 8); }
inline void tmem_store_16x8(uint32_t at, const uint32_t (&)[4]) { tmem_store(at, 8); }

struct Operand {                              // (the model goes by the address alone)
  uint32_t at;
  Operand operator+(uint32_t bytes) const { return {at + bytes}; }
};
inline Operand operand(uint32_t addr, uint32_t, uint32_t) { return {addr}; }
constexpr uint32_t mma_bf16(int, int, bool, bool) { return 0; }
void mma_ss(uint32_t d, Operand a, Operand b, uint32_t what, bool add);
void mma_ts(uint32_t d, uint32_t a, Operand b, uint32_t what, bool add);
template <bool ADD> void mma_ss(uint32_t d, Operand a, Operand b, uint32_t what) { mma_ss(d, a, b, what, ADD); }
template <bool ADD> void mma_ts(uint32_t d, uint32_t a, Operand b, uint32_t what) { mma_ts(d, a, b, what, ADD); }
void mma_commit(uint32_t bar);

inline uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  uint32_t r;
  memcpy(&r, &p, 4);
  return r;
}
inline float exp2_fast(float x) { return exp2f(x); }

}  // namespace lq
