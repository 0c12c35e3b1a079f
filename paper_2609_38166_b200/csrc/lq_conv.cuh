// Short causal depthwise convolution with SiLU: packed prompts and single tokens.
//
// out[t][c] = f(bias[c] + sum_i w[c][i] x[t-(width-1)+i][c]): two multiply-adds a tap and one exponential per element, against
// 2 x 2 bytes of traffic - bound by memory.  A thread owns VEC neighbouring channels (four; one where
// their number, strides or addresses do not divide) and walks down the rows of its
// tile with the last width-1 rows in registers, so a row is read once per tile (and width-1 rows of the tile before it).
// 32768 rows x 8192 channels: bf16 191 us, 5.6 TB/s (the exponential and the quotient alone are 119 us of the special-function units; 253 us
// with elements taken apart and rounded one by one, 360 with eight channels to a thread, which leave room for fewer warps); 16384 rows in
// binary32 183 us, 5.9 TB/s.
//
// exp and the quotient are the approximate ones: off by 2^-22 and 2^-23 of themselves, next to the |y| 2^-23 that the exponent's rounding to binary32
// costs in any case.  The exact ones are several instructions more for each element.  Where exp(-y) is 2^126 or more (y below -87.3) the quotient is 0.
#pragma once
#include "lq_rows.cuh"

namespace lq {

struct ConvArgs {
  const void *x, *w, *bias;
  void *state, *out;
  int64_t x_stride, out_stride;
  Sequences sq;
  int channels, silu, rows_per_tile, blocks_c;   // blocks_c: CTAs side by side in a row
};

constexpr int CONV_THREADS = 128;

__device__ __forceinline__ float exp2_ftz(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// VEC values in binary32, as pairs where VEC is even: sums go two channels at a time.
template <int VEC>
struct ConvRow {
  float x[VEC];
  // x + a * b, channel by channel
  __device__ __forceinline__ void add(const ConvRow &a, const ConvRow &b) {
    if constexpr (VEC % 2 == 0) {
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 s = __ffma2_rn(make_float2(a.x[e], a.x[e + 1]), make_float2(b.x[e], b.x[e + 1]), make_float2(x[e], x[e + 1]));
        x[e] = s.x;
        x[e + 1] = s.y;
      }
    } else {
      x[0] = fmaf(a.x[0], b.x[0], x[0]);
    }
  }
};

// The taps of a thread's channels and the sum over them, in binary32.
template <typename T, int W, int VEC>
struct ConvTaps {
  ConvRow<VEC> w[W], bias;
  int silu;
  __device__ __forceinline__ void load(const ConvArgs &a, int c) {
    const T *src = static_cast<const T *>(a.w) + (size_t)c * W;
    alignas(16) T t[VEC * W];
    load_row<VEC != 1>(src, t);
#pragma unroll
    for (int e = 0; e < VEC; e++)
#pragma unroll
      for (int i = 0; i < W; i++) w[i].x[e] = to_float(t[e * W + i]);
#pragma unroll
    for (int e = 0; e < VEC; e++) bias.x[e] = a.bias ? to_float(static_cast<const T *>(a.bias)[c + e]) : 0.0f;
    silu = a.silu;
  }
  // rows[i] is the row that tap i meets
  __device__ __forceinline__ void apply(const ConvRow<VEC> *rows, T (&y)[VEC]) const {
    ConvRow<VEC> s = bias;
#pragma unroll
    for (int i = 0; i < W; i++) s.add(w[i], rows[i]);
    if (silu) {                               // y / (1 + exp(-y)): a quotient that overflows is a product with 0
#pragma unroll
      for (int e = 0; e < VEC; e++) s.x[e] *= reciprocal(1.0f + exp2_ftz(s.x[e] * -1.44269504088896340736f));
    }
    pack(s.x, y);
  }
};

template <typename T, int W, int VEC>
__global__ void __launch_bounds__(CONV_THREADS) conv_prompt_kernel(const ConvArgs a) {
  constexpr int H = W - 1, U = 8;             // rows of history; rows on their way while as many are worked on
  constexpr bool WIDE = VEC != 1;
  const Sequences &sq = a.sq;
  // (CTAs that run at the same time have whole rows between them: neighbouring pieces of memory)
  const int tile = blockIdx.x / a.blocks_c, c = ((blockIdx.x - tile * a.blocks_c) * CONV_THREADS + threadIdx.x) * VEC;
  // A tile whose border falls on one of the first rows of a sequence but its very first leaves these to the tile in front of it: the
  // slot is read and written by the tile that has a sequence's first row, and no other tile looks at it.
  auto border = [&](int t, int n) {
    if (n < 0 || n >= sq.seqs) return t;
    const int s = sq.first(n), e = sq.first(n + 1);
    return t > s && t < s + H ? max(t, min(s + H, e)) : t;
  };
  const int t0 = tile * a.rows_per_tile, t1 = min(t0 + a.rows_per_tile, sq.tokens);
  const int2 at = sequences_at(sq, t0, t1);
  int n = at.x, t = border(t0, at.x);
  const int end = t1 < sq.tokens ? border(t1, at.y) : t1;
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
    ConvRow<VEC> rows[W];                     // the rows that the taps meet, in binary32
#pragma unroll
    for (int i = 0; i < H; i++) unpack(hist[i], rows[i + 1].x);
    alignas(16) T next[U][VEC];
    const T *in = x + from * a.x_stride;
    T *to_row = out + from * a.out_stride;
    // the next rows from `first` on; where all of them are there, without a question for each
    auto load = [&](int first) {
      if (first + U <= to) {
#pragma unroll
        for (int i = 0; i < U; i++) load_row<WIDE>(in + i * a.x_stride, next[i]);
      } else {
#pragma unroll
        for (int i = 0; i < U; i++)
          if (first + i < to) load_row<WIDE>(in + i * a.x_stride, next[i]);
      }
      in += U * a.x_stride;
    };
    load(from);
#pragma unroll 1
    for (int r = from; r < to; r += U) {
      alignas(16) T now[U][VEC];
#pragma unroll
      for (int i = 0; i < U; i++)
#pragma unroll
        for (int v = 0; v < VEC; v++) now[i][v] = next[i][v];
      load(r + U);
      const bool all = r + U <= to;
#pragma unroll
      for (int i = 0; i < U; i++) {
#pragma unroll
        for (int k = 0; k < H; k++) rows[k] = rows[k + 1];
        unpack(now[i], rows[H].x);
        alignas(16) T y[VEC];
        taps.apply(rows, y);
        if (all || r + i < to) store_row<WIDE>(to_row + i * a.out_stride, y);
      }
      to_row += U * a.out_stride;
    }
  }
}

// One row per sequence.  out may be x: a thread reads its channels before it writes them.
template <typename T, int W, int VEC>
__global__ void __launch_bounds__(CONV_THREADS) conv_step_kernel(const ConvArgs a) {
  constexpr int H = W - 1;
  constexpr bool WIDE = VEC != 1;
  const int n = blockIdx.x / a.blocks_c, c = ((blockIdx.x - n * a.blocks_c) * CONV_THREADS + threadIdx.x) * VEC;
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
  ConvRow<VEC> x[W];
#pragma unroll
  for (int i = 0; i < W; i++) unpack(rows[i], x[i].x);
  taps.apply(x, y);
  store_row<WIDE>(static_cast<T *>(a.out) + n * a.out_stride + c, y);
#pragma unroll
  for (int i = 0; i < H; i++) store_row<WIDE>(state + (size_t)i * a.channels, rows[i + 1]);
}

}  // namespace lq
