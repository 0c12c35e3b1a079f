// What lq_scan.cuh needs of CUDA to be compiled for the host, where a warp is one fiber that stands for its lane 0 (see scan_roles.cpp).
#pragma once
#include <math.h>
#include <string.h>

#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#undef __device__
#undef __global__
#undef __forceinline__
#undef __launch_bounds__
#undef __shared__
#undef __align__
#undef __grid_constant__
#define __device__
#define __global__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
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

void yield();                                 // somebody else may go on here
void cta_barrier();

inline void __syncwarp() { yield(); }
inline void __syncthreads() { cta_barrier(); }
inline int __syncthreads_count(int) { abort(); }
inline bool __all_sync(unsigned, bool p) { return p; }
template <typename T> inline T __shfl_sync(unsigned, T x, int) { return x; }
template <typename T> inline T __shfl_up_sync(unsigned, T x, int) { return x; }
inline int atomicAdd(int *p, int x) { const int old = *p; *p += x; return old; }
inline int atomicOr(int *p, int x) { const int old = *p; *p |= x; return old; }
inline float __uint_as_float(unsigned x) { float f; memcpy(&f, &x, 4); return f; }
inline unsigned __float_as_uint(float f) { unsigned x; memcpy(&x, &f, 4); return x; }
inline unsigned __byte_perm(unsigned, unsigned, unsigned) { return 0; }
inline float2 __fmul2_rn(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }
inline float2 __fadd2_rn(float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }
inline float2 __ffma2_rn(float2 a, float2 b, float2 c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }
