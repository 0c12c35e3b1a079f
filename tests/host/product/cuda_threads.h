// What lq_product.cuh needs of CUDA to be compiled for the host, where a thread is a fiber (see product_roles.cpp).
#pragma once
#include <math.h>
#include <string.h>

#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#undef __device__
#undef __global__
#undef __forceinline__
#undef __launch_bounds__
#undef __cluster_dims__
#undef __shared__
#undef __align__
#undef __grid_constant__
#define __device__
#define __global__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __cluster_dims__(...)
#define __shared__
#define __align__(n) __attribute__((aligned(n)))
#define __grid_constant__
#define PTX(...)                              // an instruction that the model does without

using std::max;
using std::min;

struct Dim {
  unsigned x;
};
extern Dim threadIdx, blockIdx, gridDim, blockDim;   // of the fiber that runs

uint8_t *cta_memory();                        // the dynamic shared memory of the CTA that runs
void yield();                                 // somebody else may go on here
void cta_barrier();
const uint64_t *warp_values(uint64_t mine);   // of all lanes, when the last of them is here

inline void __syncwarp() { warp_values(0); }
inline void __syncthreads() { cta_barrier(); }
inline int __syncthreads_count(int) { abort(); }
inline bool __any_sync(unsigned, bool p) {
  const uint64_t *v = warp_values(p);
  return std::any_of(v, v + 32, [](uint64_t x) { return x != 0; });
}
inline bool __all_sync(unsigned m, bool p) { return !__any_sync(m, !p); }
inline int __shfl_sync(unsigned, int x, int lane) { return (int)warp_values((uint32_t)x)[lane]; }
inline int __shfl_up_sync(unsigned, int x, int by) {
  const uint64_t *v = warp_values((uint32_t)x);
  const int lane = threadIdx.x % 32;
  return lane >= by ? (int)v[lane - by] : x;
}
inline int atomicOr(int *p, int x) { const int old = *p; *p |= x; return old; }
inline float __uint_as_float(unsigned x) { float f; memcpy(&f, &x, 4); return f; }
inline unsigned __float_as_uint(float f) { unsigned x; memcpy(&x, &f, 4); return x; }
inline float2 __ffma2_rn(float2 a, float2 b, float2 c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }
inline unsigned two_bf16(float lo, float hi) {
  const __nv_bfloat16 t[2] = {__float2bfloat16_rn(lo), __float2bfloat16_rn(hi)};
  unsigned r;
  memcpy(&r, t, 4);
  return r;
}
inline unsigned two_f16(float lo, float hi) {
  const __half t[2] = {__float2half_rn(lo), __float2half_rn(hi)};
  unsigned r;
  memcpy(&r, t, 4);
  return r;
}
