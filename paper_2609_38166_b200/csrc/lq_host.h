// What the entry points of the operators on packed rows share on the host: checks of arguments, the driver's tensor maps.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "../../include/lq.h"

namespace lq {

inline cudaStream_t cuda_stream(lq_stream s) { return reinterpret_cast<cudaStream_t>(s); }

inline bool aligned(const void *p, unsigned bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

inline lq_status launched() { return cudaGetLastError() == cudaSuccess ? LQ_OK : LQ_ERR_CUDA; }

inline unsigned type_size(int type) { return type == LQ_F32 ? 4 : 2; }

inline long ceil_div(long a, long b) { return (a + b - 1) / b; }

inline bool bad_count(int n) { return n < 0; }

// Row and sequence numbers up to a tile or a CTA beyond the last one are formed in 32 bits.
constexpr int MOST_ROWS = INT32_MAX - 1023;

// Required and optional (may be null) arrays with elements of `bytes` bytes.
inline lq_status check_arrays(unsigned bytes, std::initializer_list<const void *> required, std::initializer_list<const void *> optional = {}) {
  for (const void *p : required) {
    if (!p) return LQ_ERR_NULL;
    if (!aligned(p, bytes)) return LQ_ERR_ALIGN;
  }
  for (const void *p : optional)
    if (!aligned(p, bytes)) return LQ_ERR_ALIGN;
  return LQ_OK;
}

// Whether two arrays of strided rows have an element in common.  Exact where the strides are equal (slices of one buffer), else
// by the ranges they span.
inline bool rows_overlap(const void *a, int64_t sa, long wa, const void *b, int64_t sb, long wb, long rows, unsigned bytes) {
  if (rows <= 0) return false;
  const intptr_t x = reinterpret_cast<intptr_t>(a), y = reinterpret_cast<intptr_t>(b);
  const intptr_t ex = x + ((rows - 1) * sa + wa) * (intptr_t)bytes, ey = y + ((rows - 1) * sb + wb) * (intptr_t)bytes;
  if (ex <= y || ey <= x) return false;
  if (sa != sb) return true;
  const intptr_t period = sa * (intptr_t)bytes, d = ((y - x) % period + period) % period;   // b's rows start d bytes into a's
  return d < wa * (intptr_t)bytes || d + wb * (intptr_t)bytes > period;
}

// Whether `bytes` bytes at p, without gaps, meet the range of those strided rows.
inline bool meets_rows(const void *p, uint64_t bytes, const void *a, int64_t sa, long wa, long rows, unsigned size) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(a);
  return rows > 0 && x < y + ((rows - 1) * (uint64_t)sa + wa) * size && y < x + bytes;
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
    cudaGetLastError();
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

}  // namespace lq
