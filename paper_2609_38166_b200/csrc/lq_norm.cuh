// Queries and keys normalised per head and rotated by position, in one pass.
//
// Every row is read and written once; the arithmetic (one sum of squares per head, four multiply-adds per rotated pair) is far below
// that - bound by memory.  A lane owns eight neighbouring channels, dim/8 neighbouring lanes a head: the sum of
// squares is a butterfly over them, and the other half of a rotated pair is one exchange away.  A CTA takes the angles of its rows
// once for all heads: position * inv_freq in binary64, brought to a fraction of a turn there, so that what binary32 gets
// is below one half whatever the position.
#pragma once
#include "lq_rows.cuh"

namespace lq {

struct NormArgs {
  const void *q, *k;
  void *out_q, *out_k;
  int64_t q_stride, k_stride, out_q_stride, out_k_stride;
  const float *w_q, *w_k, *inv_freq;
  const int32_t *positions;
  int tokens, heads_q, heads_k, rot, pairs, norm, rows_per_cta;
  float eps, scale_q, scale_k;
};

constexpr int NORM_THREADS = 256;
constexpr int NORM_MAX_ROWS = 4;              // rows of a CTA

template <typename T, int DIM, bool WIDE>
__global__ void __launch_bounds__(NORM_THREADS) norm_rotate_kernel(const NormArgs a) {
  constexpr int LANES = DIM / 8;              // of a head
  __shared__ float2 turn[NORM_MAX_ROWS][DIM / 2];
  const int row0 = blockIdx.x * a.rows_per_cta, rows = min(a.rows_per_cta, a.tokens - row0);
  const int half = a.rot / 2, heads = a.heads_q + a.heads_k;
  if (half > 0) {
    for (int i = threadIdx.x; i < rows * half; i += NORM_THREADS) {
      const int r = i / half, f = i - r * half;
      const double turns = (double)a.positions[row0 + r] * (double)a.inv_freq[f] * 0.15915494309189533577;   // / (2 pi)
      float sn, cs;
      sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
      turn[r][f] = make_float2(cs, sn);
    }
    __syncthreads();
  }
  const int lane = threadIdx.x % LANES, c = 8 * lane;
  const int units = rows * heads;             // heads of all rows
#pragma unroll 1
  for (int u0 = threadIdx.x / 32 * (32 / LANES); u0 < units; u0 += NORM_THREADS / LANES) {   // (the same trips for all lanes of a warp)
    const int u = u0 + threadIdx.x % 32 / LANES;
    const bool there = u < units;
    const int r = there ? u / heads : 0, h = there ? u - r * heads : 0;
    const bool is_q = h < a.heads_q;
    const int64_t row = row0 + r;
    const T *src = is_q ? static_cast<const T *>(a.q) + row * a.q_stride + h * DIM
                        : static_cast<const T *>(a.k) + row * a.k_stride + (h - a.heads_q) * DIM;
    alignas(16) T in[8];
#pragma unroll
    for (int e = 0; e < 8; e++) in[e] = from_float<T>(0.0f);
    if (there) load_row<WIDE>(src + c, in);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = to_float(in[e]);
    float scale = is_q ? a.scale_q : a.scale_k;
    if (a.norm != LQ_NORM_NONE) {
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; e++) s = fmaf(x[e], x[e], s);
#pragma unroll
      for (int m = 1; m < LANES; m *= 2) s += __shfl_xor_sync(0xffffffffu, s, m);
      scale *= rsqrtf((a.norm == LQ_NORM_RMS ? s * (1.0f / DIM) : s) + a.eps);
    }
    const float *w = is_q ? a.w_q : a.w_k;
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] *= scale * (a.norm == LQ_NORM_RMS && w ? w[c + e] : 1.0f);
    if (a.pairs) {
      if (c < a.rot) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float2 t = turn[r][(c + e) / 2];
          const float y0 = x[e], y1 = x[e + 1];
          x[e] = fmaf(y0, t.x, -(y1 * t.y));
          x[e + 1] = fmaf(y1, t.x, y0 * t.y);
        }
      }
    } else if (half > 0) {                    // the other half of a pair sits half/8 lanes further or back
      const bool low = c < half;
      const int other = low ? lane + half / 8 : lane - half / 8;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float y = __shfl_sync(0xffffffffu, x[e], other & (LANES - 1), LANES);
        if (c < a.rot) {
          const float2 t = turn[r][(low ? c : c - half) + e];
          x[e] = low ? fmaf(x[e], t.x, -(y * t.y)) : fmaf(x[e], t.x, y * t.y);
        }
      }
    }
    if (there && (!a.positions || a.positions[row] >= 0)) {
      alignas(16) T y[8];
#pragma unroll
      for (int e = 0; e < 8; e++) y[e] = from_float<T>(x[e]);
      T *dst = is_q ? static_cast<T *>(a.out_q) + row * a.out_q_stride + h * DIM
                    : static_cast<T *>(a.out_k) + row * a.out_k_stride + (h - a.heads_q) * DIM;
      store_row<WIDE>(dst + c, y);
    }
  }
}

}  // namespace lq
