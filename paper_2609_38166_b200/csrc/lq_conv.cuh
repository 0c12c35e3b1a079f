// Short causal depthwise convolution with SiLU: packed prompts and single tokens.
//
// out[t][c] = f(bias[c] + sum_i w[c][i] x[t-(width-1)+i][c]): two multiply-adds a tap and one exponential per element, against
// 2 x 2 bytes of traffic - bound by memory.  A thread owns VEC neighbouring channels (16 bytes) and walks down the rows of its
// tile with the last width-1 rows in registers, so a row is read once per tile (and width-1 rows of the tile before it).
#pragma once
#include "lq_rows.cuh"

namespace lq {

struct ConvArgs {
  const void *x, *w, *bias;
  void *state, *out;
  int64_t x_stride, out_stride;
  Sequences sq;
  int channels, silu, rows_per_tile;
};

constexpr int CONV_THREADS = 128;

// The taps of a thread's channels and the sum over them, in binary32.
template <typename T, int W, int VEC>
struct ConvTaps {
  float w[W][VEC], bias[VEC];
  int silu;
  __device__ __forceinline__ void load(const ConvArgs &a, int c) {
    const T *src = static_cast<const T *>(a.w) + (size_t)c * W;
    alignas(16) T t[VEC * W];
    load_row<VEC != 1>(src, t);
#pragma unroll
    for (int e = 0; e < VEC; e++)
#pragma unroll
      for (int i = 0; i < W; i++) w[i][e] = to_float(t[e * W + i]);
#pragma unroll
    for (int e = 0; e < VEC; e++) bias[e] = a.bias ? to_float(static_cast<const T *>(a.bias)[c + e]) : 0.0f;
    silu = a.silu;
  }
  // rows[i] is the row that tap i meets
  __device__ __forceinline__ void apply(const T (&r0)[VEC], const T (*hist)[VEC], T (&y)[VEC]) const {
#pragma unroll
    for (int e = 0; e < VEC; e++) {
      float s = bias[e];
#pragma unroll
      for (int i = 0; i < W - 1; i++) s = fmaf(w[i][e], to_float(hist[i][e]), s);
      s = fmaf(w[W - 1][e], to_float(r0[e]), s);
      if (silu) s = __fdividef(s, 1.0f + __expf(-s));
      y[e] = from_float<T>(s);
    }
  }
};

template <typename T, int W, int VEC>
__global__ void __launch_bounds__(CONV_THREADS) conv_prompt_kernel(const ConvArgs a) {
  constexpr int H = W - 1, U = 8;             // rows of history; rows in flight
  constexpr bool WIDE = VEC != 1;
  const Sequences &sq = a.sq;
  const int c = (blockIdx.y * CONV_THREADS + threadIdx.x) * VEC;
  // A tile whose border falls on one of the first rows of a sequence but its very first leaves these to the tile in front of it: the
  // slot is read and written by the tile that has a sequence's first row, and no other tile looks at it.
  auto border = [&](int t, int n) {
    if (n < 0 || n >= sq.seqs) return t;
    const int s = sq.first(n), e = sq.first(n + 1);
    return t > s && t < s + H ? max(t, min(s + H, e)) : t;
  };
  const int t0 = blockIdx.x * a.rows_per_tile, t1 = min(t0 + a.rows_per_tile, sq.tokens);
  int n = sequence_at(sq, t0);
  const int n1 = t1 < sq.tokens ? sequence_at(sq, t1) : -1;
  int t = border(t0, n);
  const int end = border(t1, n1);
  if (c >= a.channels) return;
  ConvTaps<T, W, VEC> taps;
  taps.load(a, c);
  const T *x = static_cast<const T *>(a.x) + c;
  T *out = static_cast<T *>(a.out) + c;
  T *state = a.state ? static_cast<T *>(a.state) + c : nullptr;
  if (n < 0) n = 0;
#pragma unroll 1
  for (; n < sq.seqs && t < end; n++) {
    const int s = sq.first(n), e = sq.first(n + 1);
    const int from = max(t, s), to = min(e, end);
    if (from >= to) continue;
    t = to;
    const int slot = sq.slot(n);
    if (slot < 0) continue;
    T *mine = state ? state + (size_t)slot * H * a.channels : nullptr;
    alignas(16) T hist[H][VEC];
#pragma unroll
    for (int i = 0; i < H; i++) {
#pragma unroll
      for (int v = 0; v < VEC; v++) hist[i][v] = from_float<T>(0.0f);
      if (from - H >= s) load_row<WIDE>(x + (from - H + i) * a.x_stride, hist[i]);
      else if (mine && sq.resumed(n)) load_row<WIDE>(mine + (size_t)i * a.channels, hist[i]);
    }
    if (from == s && mine) {                  // the last H rows of (old state, x) are the new state
#pragma unroll
      for (int j = 0; j < H; j++) {
        const int r = e - H + j;
        alignas(16) T last[VEC];
        if (r >= s) {
          load_row<WIDE>(x + r * a.x_stride, last);
        } else {
#pragma unroll
          for (int v = 0; v < VEC; v++) {
            last[v] = hist[0][v];
#pragma unroll
            for (int i = 1; i < H; i++)
              if (i == H + r - s) last[v] = hist[i][v];
          }
        }
        store_row<WIDE>(mine + (size_t)j * a.channels, last);
      }
    }
#pragma unroll 1
    for (int r = from; r < to; r += U) {
      alignas(16) T rows[H + U][VEC];
#pragma unroll
      for (int i = 0; i < H; i++)
#pragma unroll
        for (int v = 0; v < VEC; v++) rows[i][v] = hist[i][v];
#pragma unroll
      for (int i = 0; i < U; i++)
        if (r + i < to) load_row<WIDE>(x + (int64_t)(r + i) * a.x_stride, rows[H + i]);
#pragma unroll
      for (int i = 0; i < U; i++)
        if (r + i < to) {
          alignas(16) T y[VEC];
          taps.apply(rows[H + i], rows + i, y);
          store_row<WIDE>(out + (int64_t)(r + i) * a.out_stride, y);
        }
#pragma unroll
      for (int i = 0; i < H; i++)
#pragma unroll
        for (int v = 0; v < VEC; v++) hist[i][v] = rows[U + i][v];
    }
  }
}

// One row per sequence.  out may be x: a thread reads its channels before it writes them.
template <typename T, int W, int VEC>
__global__ void __launch_bounds__(CONV_THREADS) conv_step_kernel(const ConvArgs a) {
  constexpr int H = W - 1;
  constexpr bool WIDE = VEC != 1;
  const int c = (blockIdx.y * CONV_THREADS + threadIdx.x) * VEC, n = blockIdx.x;
  const int slot = a.sq.slot(n);
  if (c >= a.channels || slot < 0) return;
  T *state = static_cast<T *>(a.state) + (size_t)slot * H * a.channels + c;
  alignas(16) T rows[W][VEC];
  alignas(16) T y[VEC];
#pragma unroll
  for (int i = 0; i < H; i++) load_row<WIDE>(state + (size_t)i * a.channels, rows[i]);
  load_row<WIDE>(static_cast<const T *>(a.x) + n * a.x_stride + c, rows[H]);
  ConvTaps<T, W, VEC> taps;
  taps.load(a, c);
  taps.apply(rows[H], rows, y);
  store_row<WIDE>(static_cast<T *>(a.out) + n * a.out_stride + c, y);
#pragma unroll
  for (int i = 0; i < H; i++) store_row<WIDE>(state + (size_t)i * a.channels, rows[i + 1]);
}

}  // namespace lq
