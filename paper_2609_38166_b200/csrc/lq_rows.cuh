// What the operators on packed rows share: element types, wide loads and stores, the sequences of a packed batch.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/lq.h"

namespace lq {

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// N consecutive elements at `src`; with WIDE in pieces of 16 or 8 bytes, to which src and N * sizeof(T) are aligned.
template <bool WIDE, typename T, int N>
__device__ __forceinline__ void load_row(const T *src, T (&x)[N]) {
  constexpr int BYTES = N * sizeof(T);
  if constexpr (WIDE && BYTES % 16 == 0) {
#pragma unroll
    for (int i = 0; i < BYTES / 16; i++) reinterpret_cast<uint4 *>(x)[i] = reinterpret_cast<const uint4 *>(src)[i];
  } else if constexpr (WIDE) {
    static_assert(BYTES % 8 == 0, "");
#pragma unroll
    for (int i = 0; i < BYTES / 8; i++) reinterpret_cast<uint2 *>(x)[i] = reinterpret_cast<const uint2 *>(src)[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = src[i];
  }
}
template <bool WIDE, typename T, int N>
__device__ __forceinline__ void store_row(T *dst, const T (&x)[N]) {
  constexpr int BYTES = N * sizeof(T);
  if constexpr (WIDE && BYTES % 16 == 0) {
#pragma unroll
    for (int i = 0; i < BYTES / 16; i++) reinterpret_cast<uint4 *>(dst)[i] = reinterpret_cast<const uint4 *>(x)[i];
  } else if constexpr (WIDE) {
#pragma unroll
    for (int i = 0; i < BYTES / 8; i++) reinterpret_cast<uint2 *>(dst)[i] = reinterpret_cast<const uint2 *>(x)[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) dst[i] = x[i];
  }
}

// N elements in binary32; pairs of bf16 by a shift and a mask of the register that they share (one by one they take twice the instructions).
template <typename T, int N>
__device__ __forceinline__ void unpack(const T (&t)[N], float (&x)[N]) {
  if constexpr (sizeof(T) == 2 && N % 2 == 0) {
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const uint32_t two = *reinterpret_cast<const uint32_t *>(&t[e]);
      if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        x[e] = __uint_as_float(two << 16);
        x[e + 1] = __uint_as_float(two & 0xFFFF0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&two));
        x[e] = f.x;
        x[e + 1] = f.y;
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; e++) x[e] = to_float(t[e]);
  }
}
// The same, rounded to T (nearest even).
template <typename T, int N>
__device__ __forceinline__ void pack(const float (&x)[N], T (&t)[N]) {
  if constexpr (sizeof(T) == 2 && N % 2 == 0) {
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      uint32_t two;
      if constexpr (std::is_same_v<T, __nv_bfloat16>) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(two) : "f"(x[e + 1]), "f"(x[e]));
      else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(two) : "f"(x[e + 1]), "f"(x[e]));
      *reinterpret_cast<uint32_t *>(&t[e]) = two;
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; e++) t[e] = from_float<T>(x[e]);
  }
}

// Division of numbers below 2^31 by a constant of the call: a multiplication and a shift.
struct Divisor {
  uint32_t d, m, shift;
  void set(uint32_t by) {
    d = by;
    shift = 0;
    while (((uint64_t)1 << shift) < by) shift++;
    m = (uint32_t)((((uint64_t)1 << (31 + shift)) + by - 1) / by);   // below 2^32
  }
  __device__ __forceinline__ uint32_t quotient(uint32_t x) const { return (uint32_t)(((uint64_t)x * m) >> 31) >> shift; }
};

// The sequences of a packed batch.  What the arrays hold is not checked by the host, so every row number is brought into
// [0, tokens] and every slot is compared with n_slots here: nothing outside of the arrays is touched whatever they hold.
struct Sequences {
  const int32_t *start, *slots, *resume;
  int tokens, seqs, n_slots;

  __device__ __forceinline__ int first(int n) const { return min(max(start[n], 0), tokens); }
  // slot of sequence n, or -1 where it is padding
  __device__ __forceinline__ int slot(int n) const {
    const int s = slots ? slots[n] : n;
    return s >= 0 && s < n_slots ? s : -1;
  }
  __device__ __forceinline__ bool resumed(int n) const { return resume && resume[n] != 0; }
};

// The last sequences that start at row t or before it and at row u or before it (-1: none), found by all threads of the CTA together.
__device__ __forceinline__ int2 sequences_at(const Sequences &sq, int t, int u) {
  int2 n = make_int2(-1, -1);
  for (int i = 0; i <= sq.seqs; i += blockDim.x) {
    const int at = i + threadIdx.x, first = at <= sq.seqs ? sq.first(at) : INT32_MAX;
    n.x += __syncthreads_count(first <= t);
    n.y += __syncthreads_count(first <= u);
  }
  return n;
}

}  // namespace lq
