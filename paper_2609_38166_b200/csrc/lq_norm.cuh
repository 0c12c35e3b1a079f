// Queries and keys normalised per head and rotated by position, in one pass.
//
// Every row is read and written once; the arithmetic (one sum of squares per head, four multiply-adds per rotated pair) is far below
// that - bound by memory.  A lane owns two 16-byte pieces of a head and neighbouring lanes the rest; the sum of squares is a butterfly over them.
// Where channels i and i + rot/2 are a pair, a lane's pieces are one of either half, so that its pairs are its own.  A CTA takes the angles of its
// rows once for all heads: a frequency in turns as a fraction of 64 bits (from binary64), times the position modulo one turn - whole
// turns drop out exactly, and what binary32 gets is at most half a turn whatever the position.
// What sincospif gets is a phase of 32 bits, as binary32: off by 2^-25 of a half turn at most.
// 16384 rows of 40 heads of 128 bf16 channels, 64 of them rotated: 64 us, 5.2 TB/s (115 us with one row to a CTA, angles in binary64 and
// partners exchanged between lanes; half the arithmetic instructions, two channels each, took as long: it is the memory's latency and
// the call's start and end that are left); all 128 rotated, in binary32, 125 us, 5.4 TB/s.
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
  Divisor heads, half;
};

constexpr int NORM_THREADS = 256;
constexpr int NORM_MAX_ROWS = 16;             // rows of a CTA
constexpr int NORM_TRIPS = 10;                // heads that a lane has in turn (16384 rows of 40 heads: 16 rows to a CTA 76 us, 8 rows 72, 4 rows 74, 1 row 117)

template <typename T, int DIM, bool WIDE>
__global__ void __launch_bounds__(NORM_THREADS, 3) norm_rotate_kernel(const NormArgs a) {
  constexpr int F = 16 / sizeof(T), LANES = DIM / (2 * F);   // channels of a piece, lanes of a head
  // by lane, 16 bytes at a time: neighbouring lanes read neighbouring pieces
  __shared__ __align__(16) float2 turn[NORM_MAX_ROWS][F / 2][LANES][2];
  __shared__ __align__(16) float weight[2][2 * F / 4][LANES][4];
  __shared__ uint64_t step[DIM / 2];
  __shared__ float nothing[DIM / 2];          // 0, or NaN where a frequency is not finite: no fraction of a turn can say so
  const int row0 = blockIdx.x * a.rows_per_cta, rows = min(a.rows_per_cta, a.tokens - row0);
  const int half = a.rot / 2, heads = a.heads_q + a.heads_k;
  const int lane = threadIdx.x % LANES;
  const bool turned = 2 * F * lane < a.rot, apart = turned && !a.pairs;
  const int c0 = apart ? F * lane : 2 * F * lane, c1 = apart ? half + F * lane : c0 + F;   // where the lane's pieces start
  const int units = rows * heads;             // heads of all rows
  constexpr int SIDE = NORM_THREADS / LANES;  // heads that the CTA has at a time
  alignas(16) T next[2][F];                   // the head on its way while one is worked on
  auto load = [&](int u) {
    if (u >= units) return;
    const int r = a.heads.quotient(u), h = u - r * heads;
    const int64_t row = row0 + r;
    const T *src = h < a.heads_q ? static_cast<const T *>(a.q) + row * a.q_stride + h * DIM
                                 : static_cast<const T *>(a.k) + row * a.k_stride + (h - a.heads_q) * DIM;
    load_row<WIDE>(src + c0, next[0]);
    load_row<WIDE>(src + c1, next[1]);
  };
  const int mine = threadIdx.x / LANES;
  load(mine);                                 // (on their way while the angles are worked out)
  if (half > 0) {
    for (int f = threadIdx.x; f < half; f += NORM_THREADS) {
      const double turns = (double)a.inv_freq[f] * 0.15915494309189533577;   // of a turn a position, / (2 pi)
      step[f] = (uint64_t)(int64_t)((turns - rint(turns)) * 18446744073709551616.0);   // modulo 1, in units of 2^-64
      nothing[f] = a.inv_freq[f] * 0.0f;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * half; i += NORM_THREADS) {
      const int r = a.half.quotient(i), f = i - r * half;
      const int32_t phase = (int32_t)((step[f] * (uint64_t)(int64_t)a.positions[row0 + r]) >> 32);
      float sn, cs;
      sincospif(fmaf((float)phase, 4.656612873077392578125e-10f, nothing[f]), &sn, &cs);   // 2^-31: in half turns
      turn[r][f % F / 2][f / F][f % 2] = make_float2(cs, sn);
    }
  }
  if (a.norm == LQ_NORM_RMS)
    for (int i = threadIdx.x; i < 2 * DIM; i += NORM_THREADS) {
      const float *w = i < DIM ? a.w_q : a.w_k;
      const int l = i % DIM / (2 * F), e = i % (2 * F);
      const int channel = 2 * F * l < a.rot && !a.pairs ? (e < F ? 0 : half - F) + F * l + e : 2 * F * l + e;
      weight[i / DIM][e / 4][l][e % 4] = w ? w[channel] : 1.0f;
    }
  __syncthreads();
#pragma unroll 1
  for (int u = mine; u - mine < units; u += SIDE) {   // (the same trips for all lanes of a warp)
    alignas(16) T in[2][F];
#pragma unroll
    for (int e = 0; e < 2 * F; e++) in[e / F][e % F] = next[e / F][e % F];
    load(u + SIDE);
    const bool there = u < units;
    const int r = there ? a.heads.quotient(u) : 0, h = there ? u - r * heads : 0;
    const bool is_q = h < a.heads_q;
    const int64_t row = row0 + r;
    float x[2][F];
    unpack(in[0], x[0]);
    unpack(in[1], x[1]);
    if (!there) {                             // (a lane without a head has registers that were never loaded)
#pragma unroll
      for (int e = 0; e < 2 * F; e++) x[e / F][e % F] = 0.0f;
    }
    float scale = is_q ? a.scale_q : a.scale_k;
    if (a.norm != LQ_NORM_NONE) {
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < 2 * F; e++) s = fmaf(x[e / F][e % F], x[e / F][e % F], s);
#pragma unroll
      for (int m = 1; m < LANES; m *= 2) s += __shfl_xor_sync(0xffffffffu, s, m);
      scale *= rsqrtf((a.norm == LQ_NORM_RMS ? s * (1.0f / DIM) : s) + a.eps);
    }
    if (a.norm == LQ_NORM_RMS) {
#pragma unroll
      for (int e = 0; e < 2 * F; e += 4) {
        const float4 w = *reinterpret_cast<const float4 *>(weight[is_q ? 0 : 1][e / 4][lane]);
        x[e / F][e % F] *= scale * w.x;
        x[e / F][e % F + 1] *= scale * w.y;
        x[e / F][e % F + 2] *= scale * w.z;
        x[e / F][e % F + 3] *= scale * w.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 2 * F; e++) x[e / F][e % F] *= scale;
    }
    if (turned) {                             // pairs: neighbours in either piece, or the pieces element by element
      float cs[F], sn[F];
#pragma unroll
      for (int p = 0; p < F; p += 2) {
        const float4 t = *reinterpret_cast<const float4 *>(turn[r][p / 2][lane]);
        cs[p] = t.x, sn[p] = t.y, cs[p + 1] = t.z, sn[p + 1] = t.w;
      }
      auto rotate = [](float &p0, float &p1, float cs, float sn) {
        const float y0 = p0, y1 = p1;
        p0 = fmaf(y0, cs, -(y1 * sn));
        p1 = fmaf(y1, cs, y0 * sn);
      };
      if (a.pairs) {
#pragma unroll
        for (int p = 0; p < F; p++) rotate(x[2 * p / F][2 * p % F], x[2 * p / F][2 * p % F + 1], cs[p], sn[p]);
      } else {
#pragma unroll
        for (int p = 0; p < F; p++) rotate(x[0][p], x[1][p], cs[p], sn[p]);
      }
    }
    if (there && (!a.positions || a.positions[row] >= 0)) {
      alignas(16) T y[2][F];
      pack(x[0], y[0]);
      pack(x[1], y[1]);
      T *dst = is_q ? static_cast<T *>(a.out_q) + row * a.out_q_stride + h * DIM
                    : static_cast<T *>(a.out_k) + row * a.out_k_stride + (h - a.heads_q) * DIM;
      store_row<WIDE>(dst + c0, y[0]);
      store_row<WIDE>(dst + c1, y[1]);
    }
  }
}

}  // namespace lq
