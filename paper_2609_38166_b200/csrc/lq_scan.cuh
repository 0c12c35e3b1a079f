// Selective state space scan with a scalar decay per head: S <- alpha S + beta k v^T, o = S^T q + skip v.
#pragma once
#include "lq_rows.cuh"

namespace lq {

constexpr int SD = 128;                       // d_k = d_v

struct ScanArgs {
  const __nv_bfloat16 *q, *k, *v;
  int64_t q_stride, k_stride, v_stride, beta_stride, alpha_stride, o_stride;
  const void *beta, *alpha;
  const float *A, *dt_bias, *skip;
  float *S;
  void *o;
  Sequences sq;
  int heads_v, heads_qk, max_len, select, gates_f32;

  __device__ __forceinline__ float gate(const void *p, int64_t i) const {
    return gates_f32 ? static_cast<const float *>(p)[i] : to_float(static_cast<const __nv_bfloat16 *>(p)[i]);
  }
};

// log(1 + exp(x))
__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.0f) + log1pf(expf(-fabsf(x))); }

// A state spread over 256 threads: warp w has rows 16 w .. 16 w + 15 (key channels), a lane four columns (value channels).
struct ScanState {
  float4 s[16];
  __device__ __forceinline__ void load(const float *S, int warp, int lane) {
#pragma unroll
    for (int i = 0; i < 16; i++) s[i] = *reinterpret_cast<const float4 *>(S + (16 * warp + i) * SD + 4 * lane);
  }
  __device__ __forceinline__ void store(float *S, int warp, int lane) const {
#pragma unroll
    for (int i = 0; i < 16; i++) *reinterpret_cast<float4 *>(S + (16 * warp + i) * SD + 4 * lane) = s[i];
  }
  // one token: the update, and this warp's share of S^T q
  __device__ __forceinline__ float4 token(float alpha, const float *bk, const float *q, float4 v) {
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < 16; i++) {
      s[i].x = fmaf(bk[i], v.x, alpha * s[i].x);
      s[i].y = fmaf(bk[i], v.y, alpha * s[i].y);
      s[i].z = fmaf(bk[i], v.z, alpha * s[i].z);
      s[i].w = fmaf(bk[i], v.w, alpha * s[i].w);
      o.x = fmaf(q[i], s[i].x, o.x);
      o.y = fmaf(q[i], s[i].y, o.y);
      o.z = fmaf(q[i], s[i].z, o.z);
      o.w = fmaf(q[i], s[i].w, o.w);
    }
    return o;
  }
};

// What a token brings, in shared memory: beta k, q, v.
struct ScanToken {
  float bk[SD], q[SD], v[SD];
  float part[8][SD];
};

// alpha of row `row`; the token's vectors go to shared memory (256 threads)
__device__ __forceinline__ float scan_fetch(const ScanArgs &a, ScanToken &t, int64_t row, int h) {
  const int hq = h / (a.heads_v / a.heads_qk), tid = threadIdx.x;
  float beta = a.gate(a.beta, row * a.beta_stride + h), alpha;
  if (a.select) {
    beta = softplus(a.dt_bias ? beta + a.dt_bias[h] : beta);
    alpha = expf(beta * a.A[h]);
  } else {
    alpha = a.gate(a.alpha, row * a.alpha_stride + h);
  }
  if (tid < SD) {
    t.bk[tid] = beta * to_float(a.k[row * a.k_stride + hq * SD + tid]);
    t.q[tid] = to_float(a.q[row * a.q_stride + hq * SD + tid]);
  } else {
    t.v[tid - SD] = to_float(a.v[row * a.v_stride + h * SD + tid - SD]);
  }
  return alpha;
}

template <typename O>
__device__ __forceinline__ void scan_emit(const ScanArgs &a, ScanToken &t, float4 o, int64_t row, int h) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, tid = threadIdx.x;
  *reinterpret_cast<float4 *>(&t.part[warp][4 * lane]) = o;
  __syncthreads();
  if (tid < SD) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; w++) s += t.part[w][tid];
    if (a.skip) s = fmaf(a.skip[h], t.v[tid], s);
    static_cast<O *>(a.o)[row * a.o_stride + h * SD + tid] = from_float<O>(s);
  }
}

// One token on the dense state: 64 KB in and 64 KB out per head and a few hundred bytes besides - bound by memory.  The
// whole state of a head is asked for before anything else.
__global__ void __launch_bounds__(256) scan_step_kernel(const ScanArgs a) {
  __shared__ __align__(16) ScanToken t;
  const int n = blockIdx.x / a.heads_v, h = blockIdx.x - n * a.heads_v;
  const int slot = a.sq.slot(n), warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (slot < 0) return;
  float *S = a.S + ((size_t)slot * a.heads_v + h) * (SD * SD);
  ScanState st;
  st.load(S, warp, lane);
  const float alpha = scan_fetch(a, t, n, h);
  __syncthreads();
  const float4 o = st.token(alpha, t.bk + 16 * warp, t.q + 16 * warp, *reinterpret_cast<const float4 *>(t.v + 4 * lane));
  st.store(S, warp, lane);
  scan_emit<float>(a, t, o, n, h);
}

// The prompt, token by token: a CTA has one head of one sequence.
__global__ void __launch_bounds__(256) scan_tokens_kernel(const ScanArgs a) {
  __shared__ __align__(16) ScanToken t;
  const int n = blockIdx.x / a.heads_v, h = blockIdx.x - n * a.heads_v;
  const int slot = a.sq.slot(n), warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int first = a.sq.first(n), end = min(a.sq.first(n + 1), first + min(a.max_len, a.sq.tokens - first));
  if (slot < 0) return;
  float *S = a.S + ((size_t)slot * a.heads_v + h) * (SD * SD);
  ScanState st;
  if (a.sq.resumed(n)) {
    st.load(S, warp, lane);
  } else {
#pragma unroll
    for (int i = 0; i < 16; i++) st.s[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }
#pragma unroll 1
  for (int row = first; row < end; row++) {
    const float alpha = scan_fetch(a, t, row, h);
    __syncthreads();
    const float4 o = st.token(alpha, t.bk + 16 * warp, t.q + 16 * warp, *reinterpret_cast<const float4 *>(t.v + 4 * lane));
    scan_emit<__nv_bfloat16>(a, t, o, row, h);
    __syncthreads();
  }
  st.store(S, warp, lane);
}

}  // namespace lq
