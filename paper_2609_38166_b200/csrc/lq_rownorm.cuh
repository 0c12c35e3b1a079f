// Norms in front of a projection and behind the recurrence, with 8-bit outputs: whole rows with the residual's addition, heads with a gate.
//
// Every element is read and written once and a row (a head) stays in registers between its sum of squares and its outputs: bound by memory.  A thread
// has pieces of eight (heads: sixteen) consecutive channels, so that neighbouring lanes have a block of 128 and its largest value is a butterfly over them.
#pragma once
#include "lq_dependent.cuh"
#include "lq_rows.cuh"

namespace lq {

constexpr int LINE = 8;                       // channels of a thread's piece
constexpr float E4M3_MAX = 448.0f, LEAST_SCALE = 0x1p-100f;

// Where outputs go: rounded to the type, and / or as e4m3 codes with a scale for every 128 channels of a row.
struct NormOut {
  void *out;
  uint8_t *out8;
  float *scale;
  int64_t out_stride, out8_stride, scale_stride;
};

// Four values as e4m3, nearest even, beyond 448 as 448, the first at the lowest address.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return lo | (uint32_t)hi << 16;
}

__device__ __forceinline__ float reciprocal_of(float x) {   // within a step
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// `n` of N values at channel c of a row, of which the others are 0; all lanes of a warp together, 128 / N with the channels of a block.
template <bool WIDE, typename T, int N>
__device__ __forceinline__ void norm_store(const NormOut &o, int64_t row, int c, int n, const float (&y)[N]) {
  if (o.out && n > 0) {
    alignas(16) T t[N];
    pack(y, t);
    T *dst = static_cast<T *>(o.out) + row * o.out_stride + c;
    if (WIDE) {
      store_row<true>(dst, t);
    } else {
#pragma unroll
      for (int e = 0; e < N; e++)
        if (e < n) dst[e] = t[e];
    }
  }
  if (o.out8) {
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < N; e++) top = fmaxf(top, fabsf(y[e]));
#pragma unroll
    for (int m = 1; m < 128 / N; m *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
    const float scale = fmaxf(top * (1.0f / E4M3_MAX), LEAST_SCALE), by = reciprocal_of(scale);   // (an infinity makes all of its block NaN: 0 * inf)
    alignas(16) uint32_t code[N / 4];
#pragma unroll
    for (int e = 0; e < N / 4; e++) code[e] = pack_e4m3(y[4 * e] * by, y[4 * e + 1] * by, y[4 * e + 2] * by, y[4 * e + 3] * by);
    uint8_t *dst = o.out8 + row * o.out8_stride + c;
    if (WIDE) {
      if (n > 0) store_row<true>(dst, reinterpret_cast<const uint8_t(&)[N]>(code));
    } else {
#pragma unroll
      for (int e = 0; e < N; e++)
        if (e < n) dst[e] = (uint8_t)(code[e / 4] >> 8 * (e % 4));
    }
    if (c % 128 == 0 && n > 0) o.scale[c / 128 * o.scale_stride + row] = scale;
  }
}

// N elements, of which `n` are there and the others 0.
template <bool WIDE, typename T, int N>
__device__ __forceinline__ void norm_load(const T *src, int n, T (&t)[N]) {
  if (WIDE && n > 0) {
    load_row<true>(src, t);
  } else {
#pragma unroll
    for (int e = 0; e < N; e++) {
      t[e] = from_float<T>(0.0f);
      if (!WIDE && e < n) t[e] = src[e];
    }
  }
}

// The same for rows of any alignment: a lane has every 32nd of the warp's 32 * N channels from c on, so that neighbouring lanes still have neighbours:
// 16384 rows x 2001 channels of bf16 to 8 bits 74 us, with eight neighbours to a lane, one by one, 141.
template <typename T, int N>
__device__ __forceinline__ void norm_load_spread(const T *src, int n, int lane, T (&t)[N]) {   // n: channels from c on
#pragma unroll
  for (int e = 0; e < N; e++) {
    t[e] = from_float<T>(0.0f);
    if (32 * e + lane < n) t[e] = src[32 * e + lane];
  }
}
template <typename T, int N>
__device__ __forceinline__ void norm_store_spread(const NormOut &o, int64_t row, int c, int n, int lane, const float (&y)[N]) {
  if (o.out) {
    T *dst = static_cast<T *>(o.out) + row * o.out_stride + c;
#pragma unroll
    for (int e = 0; e < N; e++)
      if (32 * e + lane < n) dst[32 * e + lane] = from_float<T>(y[e]);
  }
  if (o.out8) {
    uint8_t *dst = o.out8 + row * o.out8_stride + c;
#pragma unroll
    for (int b = 0; b < N; b += 4) {          // a block of 128
      float top = fmaxf(fmaxf(fabsf(y[b]), fabsf(y[b + 1])), fmaxf(fabsf(y[b + 2]), fabsf(y[b + 3])));
#pragma unroll
      for (int m = 1; m < 32; m *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
      const float scale = fmaxf(top * (1.0f / E4M3_MAX), LEAST_SCALE), by = reciprocal_of(scale);
      const uint32_t code = pack_e4m3(y[b] * by, y[b + 1] * by, y[b + 2] * by, y[b + 3] * by);
#pragma unroll
      for (int e = 0; e < 4; e++)
        if (32 * (b + e) + lane < n) dst[32 * (b + e) + lane] = (uint8_t)(code >> 8 * e);
      if (lane == 0 && 32 * b < n) o.scale[(c / 128 + b / 4) * o.scale_stride + row] = scale;
    }
  }
}

// What a sum of squares makes of a norm.
__device__ __forceinline__ float norm_factor(float squares, float of, float eps) { return rsqrtf(fmaf(squares, of, eps)); }   // of: 1 / dim (RMS) or 1

// ---- whole rows: h = x + residual, y = norm(h) w ----
struct AddArgs {
  const void *x;
  void *residual;
  const float *w;
  int64_t x_stride, residual_stride;
  NormOut o;
  int tokens, dim, norm;
  float eps, of;
};

// blockDim: (threads of a row, rows).  A thread has V pieces; all of them are asked for before the first is written back: 16384 rows x 4096 channels, bf16 to
// 8 bits with the residual, 84 -> 78 us, with a reciprocal for the quotient 72, 6.5 TB/s, the measured copy rate.
template <typename T, bool WIDE, int V>
__global__ void __launch_bounds__(512) norm_add_kernel(const AddArgs a) {
  __shared__ float part[16];
  grid_dependency_wait();
  const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const bool there = row < a.tokens;
  const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
  T *r = static_cast<T *>(a.residual) + row * a.residual_stride;
  alignas(16) T raw[V][LINE], more[V][LINE];
  float h[V][LINE];
  float squares = 0.0f;
  const int lane = threadIdx.x % 32;
  // a piece's first channel (of the warp's, where it is spread), and how many are there
  auto channel = [&](int v) { return (v * (int)blockDim.x + (int)threadIdx.x - (WIDE ? 0 : lane)) * LINE; };
  auto count = [&](int v) { return there ? a.dim - channel(v) : 0; };
  auto load = [&](const auto *src, int v, auto &t) {
    if constexpr (WIDE) norm_load<true>(src + channel(v), count(v), t);
    else norm_load_spread(src + channel(v), count(v), lane, t);
  };
#pragma unroll
  for (int v = 0; v < V; v++) {
    load(x, v, raw[v]);
    if (a.residual) load(r, v, more[v]);
  }
#pragma unroll
  for (int v = 0; v < V; v++) {
    unpack(raw[v], h[v]);
    if (a.residual) {
      float y[LINE];
      unpack(more[v], y);
#pragma unroll
      for (int e = 0; e < LINE; e++) h[v][e] += y[e];
      alignas(16) T t[LINE];
      pack(h[v], t);
      if constexpr (WIDE) {
        if (count(v) > 0) store_row<true>(r + channel(v), t);
      } else {
#pragma unroll
        for (int e = 0; e < LINE; e++)
          if (32 * e + lane < count(v)) r[channel(v) + 32 * e + lane] = t[e];
      }
    }
#pragma unroll
    for (int e = 0; e < LINE; e++) squares = fmaf(h[v][e], h[v][e], squares);
  }
  float factor = 1.0f;
  if (a.norm != LQ_NORM_NONE) {
#pragma unroll
    for (int m = 1; m < 32; m *= 2) squares += __shfl_xor_sync(0xffffffffu, squares, m);
    const int warps = blockDim.x / 32, first = threadIdx.y * warps;
    if (lane == 0) part[first + threadIdx.x / 32] = squares;
    __syncthreads();
    squares = part[first];
    for (int w = 1; w < warps; w++) squares += part[first + w];
    factor = norm_factor(squares, a.of, a.eps);
  }
#pragma unroll
  for (int v = 0; v < V; v++) {
    if (a.norm == LQ_NORM_RMS && a.w) {
      float w[LINE];
      load(a.w, v, w);
#pragma unroll
      for (int e = 0; e < LINE; e++) h[v][e] *= factor * w[e];
    } else {
#pragma unroll
      for (int e = 0; e < LINE; e++) h[v][e] *= factor;
    }
    if constexpr (WIDE) norm_store<true, T>(a.o, row, channel(v), count(v), h[v]);
    else norm_store_spread<T>(a.o, row, channel(v), count(v), lane, h[v]);
  }
}

// ---- heads behind the recurrence: y = norm(o) w act(z) ----
struct GatedArgs {
  const void *x, *z;
  const float *w;
  int64_t x_stride, z_stride;
  NormOut o;
  int tokens, heads, dim, norm, silu;
  float eps, of;
  int warps;                                  // warps of a row
  Divisor by_warps;
};

constexpr int GATED_THREADS = 128, GATED_LINE = 16;   // channels of a lane

// 1 / (1 + exp(-z)), times z; a quotient that overflows is a 0.  In front of 8 and 16 bits the exponential is an approximation whose argument is rounded, 2^-21 +
// 2^-23 |z| off with the rest; where z and out are binary32 it is within 2^-22, and the whole within 2^-21 whatever z is.
template <typename T>
__device__ __forceinline__ float gate_of(float z, int silu) {
  float e;
  if constexpr (std::is_same_v<T, float>) e = expf(-z);
  else asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.44269504088896340736f));
  const float r = reciprocal_of(1.0f + e);
  return silu ? z * r : r;
}

// A warp has 512 channels of a row.  Sixteen channels to a lane, for what a lane does for all of them together (sums over lanes, scale, addresses) is as much
// as what it does for eight: 16384 rows x 32 heads x 128 channels of bf16 to 8 bits 80 -> 65 us; ten CTAs to an SM 62.6, 5.4 TB/s, of binary32 79, 5.9 TB/s (z and out of
// binary32, nine to an SM, for the registers of the other exponential: 137 us, 5.9 TB/s; ten 153).  What is
// left are two MUFU operations an element (30 us) next to the memory; four rows to a warp, or eight channels and four rows, take longer.
template <typename X, typename T, bool WIDE>
__global__ void __launch_bounds__(GATED_THREADS, sizeof(T) == 4 ? 9 : 10) norm_gate_kernel(const GatedArgs a) {
  constexpr int N = GATED_LINE;
  grid_dependency_wait();
  const int lane = threadIdx.x % 32;
  const uint32_t unit = blockIdx.x * (GATED_THREADS / 32) + threadIdx.x / 32, row = a.by_warps.quotient(unit);
  if (row >= (uint32_t)a.tokens) return;
  const int c = ((unit - row * a.warps) * 32 + lane) * N, n = c < a.heads * a.dim ? N : 0;
  alignas(16) X xs[N];
  alignas(16) T zs[N];
  norm_load<WIDE>(static_cast<const X *>(a.x) + row * a.x_stride + c, n, xs);
  norm_load<WIDE>(static_cast<const T *>(a.z) + row * a.z_stride + c, n, zs);
  float x[N], z[N];
  unpack(xs, x);
  float factor = 1.0f;
  if (a.norm != LQ_NORM_NONE) {
    float squares = 0.0f;
#pragma unroll
    for (int e = 0; e < N; e++) squares = fmaf(x[e], x[e], squares);
    for (int m = 1; m < a.dim / N; m *= 2) squares += __shfl_xor_sync(0xffffffffu, squares, m);
    factor = norm_factor(squares, a.of, a.eps);
  }
  if (a.norm == LQ_NORM_RMS && a.w) {
    float w[N];
    norm_load<WIDE>(a.w + c % a.dim, N, w);
#pragma unroll
    for (int e = 0; e < N; e++) x[e] *= w[e];
  }
  unpack(zs, z);
#pragma unroll
  for (int e = 0; e < N; e++) x[e] *= factor * gate_of<T>(z[e], a.silu);
  norm_store<WIDE, T>(a.o, row, c, n, x);
}

}  // namespace lq
