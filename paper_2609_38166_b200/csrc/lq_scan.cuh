// Selective state space scan with a scalar decay per head: S <- alpha S + beta k v^T, o = S^T q + skip v.
#pragma once
#include "lq_rows.cuh"
#include "lq_tensor.cuh"

namespace lq {

constexpr int SD = 128;                       // d_k = d_v

struct ScanArgs {
  const __nv_bfloat16 *q, *k, *v;
  int64_t q_stride, k_stride, v_stride, beta_stride, alpha_stride, o_stride;
  const void *beta, *alpha;
  const float *A, *dt_bias, *skip;
  const float *S0;                             // where resumed sequences start from; S, or another array of the same slots
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

__device__ __forceinline__ void scan_emit(const ScanArgs &a, ScanToken &t, float4 o, int64_t row, int h) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, tid = threadIdx.x;
  *reinterpret_cast<float4 *>(&t.part[warp][4 * lane]) = o;
  __syncthreads();
  if (tid < SD) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; w++) s += t.part[w][tid];
    if (a.skip) s = fmaf(a.skip[h], t.v[tid], s);
    static_cast<float *>(a.o)[row * a.o_stride + h * SD + tid] = s;
  }
}

// One token on the dense state: 64 KB in and 64 KB out per head and a few hundred bytes besides - bound by memory.  The
// whole state of a head is asked for before anything else.  8192 states: 164 us, the measured copy rate.
__global__ void __launch_bounds__(256) scan_step_kernel(const ScanArgs a) {
  __shared__ __align__(16) ScanToken t;
  const int n = blockIdx.x / a.heads_v, h = blockIdx.x - n * a.heads_v;
  const int slot = a.sq.slot(n), warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (slot < 0) return;
  const size_t at = ((size_t)slot * a.heads_v + h) * (SD * SD);
  ScanState st;
  st.load(a.S0 + at, warp, lane);
  const float alpha = scan_fetch(a, t, n, h);
  __syncthreads();
  const float4 o = st.token(alpha, t.bk + 16 * warp, t.q + 16 * warp, *reinterpret_cast<const float4 *>(t.v + 4 * lane));
  st.store(a.S + at, warp, lane);
  scan_emit(a, t, o, n, h);
}

// ---------------------------------------------------------------------------------------------
// Prompts, by blocks of C = 128 rows.  With G_i the sum of the block's log decays up to row i, P = Q K^T and S the state in front:
//     o_i = exp(G_i) S^T q_i + sum_{j <= i} exp(G_i - G_j) beta_j P_ij v_j + skip v_i
//     S   = exp(G_C) S + sum_j k_j (w_j v_j)^T,      w_j = exp(G_C - G_j) beta_j
// Four products of 128 x 128 x 128 on the tensor cores: P, S^T q, the weighted P times V, and the state's, whose weighted values are
// split into three bf16 pieces that add up to all 24 bits - the state stays binary32, at the price of three products for one.  P's
// weights and S are rounded to bf16 where they enter a product with an output that is itself rounded to bf16.
//
// Six products of 2 * 128^3 operations a block and head are 0.38 us each at what one SM has of the measured peak (0.26 us, 512 clocks, at the
// tensor pipe's own rate): 2.3 us (1.6).  The 64 KB of v and o (q and k are shared by the heads of a group and come from L2) take 1.5 us at its
// share of the bandwidth.  Both bounds are close, so everything runs side by side in one CTA per SM, every warp with one part.  Measured: 3.1 us a block where memory is quiet, 4.3 where
// all SMs load (8 prompts x 2048 rows x 32 heads: 122 us, 3.3 TB/s; the tensor pipe is active 48 % of the time).  What bounds it are the hand-overs
// between the parts and the fetching of their code.  (The compiler spills 56 bytes a thread in the instances with outputs, 40 in those without.)
//   warp 0       takes the next head and tells the others; tensor copies of the tiles of 32 KB, two slots each for K, Q and V
//   warp 1       the products for the outputs: P, S^T q, weighted P times V
//   warp 2       the block's gates: log decays, their sums, weights
//   warp 3       the product for the state, dS^T = (weighted V)^T K
//   warps 4-7    a row of P per thread: weights on P (to tensor memory, as the next product's operand)
//   warps 8-15   half a row of o per thread: the factor that both of its parts have, the skip, outputs
//   warps 16-23  weighted values (to tensor memory, 32 rows at a time, the operand of the state's product)
//   warps 24-27  a value channel of S per thread (128 registers): S <- gamma S + dS, S as bf16 to shared memory
// dS does not depend on S, so the only chain from block to block is S's update between two products.
//
// Both parts of o_i add up in one accumulator, S^T q_i + sum_j exp(-G_j) beta_j P_ij v_j, and exp(G_i) comes on in the end; where G_i is below
// -60 (of log2), the accumulator is held at 2^60 o_i instead (so that it overflows for outputs beyond 2^67 only): S^T q_i then enters with 2^-60
// rather than with less, 44 bits below what a bf16 output next to it can show.
//
// A sum G of log2 decays is held as a whole number and a fraction, added up apart: differences of sums lose nothing however far the
// sums have come (a decay of 0 counts as 2^-200).
//
// Long prompts of few heads are cut into pieces of `piece` rows: a first pass (OUT false: dS only) leaves every piece's own sum and decay in the
// workspace, scan_join_kernel turns them into the states in front of the pieces, and the second pass runs all pieces side by side.
// ---------------------------------------------------------------------------------------------
struct ScanMaps {
  CUtensorMap q, k, v;
};
struct ScanPlan {
  int piece, pieces;            // rows of a piece, pieces of the longest prompt (1: not cut)
  int items;                    // seqs * pieces * heads_v
  Divisor heads, cuts, group;   // division by heads_v, by pieces, by the value heads of a q/k head
  int *next;                    // how many items have been taken beyond the first of every CTA (null: they are dealt out in turn)
  int *order;                   // the sequences by length, the longest first (null: as they come)
  float *states, *decays;       // [seqs][pieces][heads_v][128][128]: the state in front of a piece; [seqs][pieces][heads_v]
};

constexpr int SB = 128;                        // rows of a block
constexpr int SCAN_THREADS = 896;
constexpr uint32_t TILE = SB * SD * 2;         // a tile of Q, K or V: two halves of 64 channels, rows of 128 bytes, swizzled
constexpr uint32_t HALF = TILE / 2;
// Columns of tensor memory: P, o and dS^T (binary32), and two buffers of weighted values (twice 16 rows in three pieces of bf16, 24 columns).  The weighted P,
// as bf16, takes the place of the first half of P: a thread has all of a row and has read what it overwrites.
constexpr int TM_P = 0, TM_O = 128, TM_DS = 256, TM_W = 384;

constexpr float LEAST = -60.0f;                // of G (log2) in the factor of an output

struct ScanSums {
  float minus_whole[SB], minus_frac[SB];       // -G of every row
  float beta[SB];
};
struct ScanWeights {
  float e[SB];                                 // beta_j exp(G at the end of j's 32 rows - G_j)
  float end_whole[4], end_frac[4];             // G at the end of every 32 rows
  float rest[4];                               // exp(G_C - G at the end of every 32 rows)
  float total, pad[3];                         // exp(G_C)
};
struct ScanShared {                            // (all but 24 bytes of what a CTA can have)
  uint8_t k[2][TILE], q[2][TILE], v[2][TILE];
  uint8_t s16[TILE];                           // S as bf16: rows of value channels, two halves of 64 key channels
  ScanSums sums;
  ScanWeights weights[2];
  int items[2][6];                             // h, slot, row, rows, at, flags
  uint64_t items_full[2], items_empty[2], k_full[2], k_empty[2], q_full[2], q_empty[2], v_full[2], v_empty[2], sums_full, sums_empty, weights_full[2], weights_empty[2];
  uint64_t w_full[2], w_empty[2], p_full, pw_full, o_full, o_free, ds_full, ds_free, s_full, s_empty, clean[2], drained[2];
  uint32_t tmem;
};
static_assert(sizeof(ScanShared) <= 232448, "");

__device__ int g_ops_error = 0;
constexpr int WAIT_LIMIT = 1 << 20;            // tries of a wait

// Bounded wait; false: it ran out, leave (everybody else's next wait will too).  (Short, for there are dozens of them: the kernel's speed hangs on
// how much of its code the instruction caches hold.)
__device__ __forceinline__ bool wait_one(const uint64_t &bar, uint32_t parity) {
  const uint32_t at = shared_addr(&bar);
  int left = WAIT_LIMIT;
#pragma unroll 1
  while (!bar_try(at, parity))
    if (--left == 0) return false;
  return true;
}
// The same of a warp, with one answer for all of its lanes.
__device__ __forceinline__ bool wait_for(const uint64_t &bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_one(bar, parity)); }

// What a CTA does in one turn of its loop: rows [row, row + rows) of a sequence, head h.
struct ScanItem {
  int h, slot, row, rows;                      // rows: -1 when there is nothing more to do
  int at;                                      // in the workspace: (sequence * pieces + piece) * heads_v + h
  int flags;                                   // 1: a state in front of it that is not zero; 2: the prompt's last piece
  int blocks;                                  // (of 128 rows)

  __device__ __forceinline__ bool state() const { return flags & 1; }
  __device__ __forceinline__ bool last() const { return flags & 2; }
  // false: there is nothing to do
  template <bool OUT>
  __device__ __forceinline__ bool find(const ScanArgs &a, const ScanPlan &plan, int item) {
    const int r = plan.heads.quotient(item), m = plan.cuts.quotient(r), n = plan.order ? plan.order[m] : m, part = r - m * plan.pieces;
    h = item - r * a.heads_v;
    at = (n * plan.pieces + part) * a.heads_v + h;
    slot = a.sq.slot(n);
    const int start = a.sq.first(n), len = min(max(a.sq.first(n + 1) - start, 0), a.max_len);
    const int from = part * plan.piece;        // (pieces * piece is less than max_len + piece)
    rows = max(min(len - from, plan.piece), 0);
    row = start + from;
    const bool end = from + rows >= len;
    flags = (OUT && (part > 0 || a.sq.resumed(n)) ? 1 : 0) | (end ? 2 : 0);
    if (slot < 0) return false;
    return OUT ? rows > 0 || part == 0 : rows > 0 && !end;
  }
};

// A thread's value channel of S (binary32) from or to global memory [128][128]: the lanes of a warp have neighbouring value channels, so
// every access is a whole line.
__device__ __forceinline__ void load_state(float (&S)[SD], const float *mem) {
#pragma unroll
  for (int j = 0; j < SD; j++) S[j] = mem[j * SD];
}
__device__ __forceinline__ void store_state(const float (&S)[SD], float *mem) {
#pragma unroll
  for (int j = 0; j < SD; j++) mem[j * SD] = S[j];
}

// A thread's value channel of S as bf16 to shared memory, where the product with q reads it.  `at`: the thread's row.
__device__ __forceinline__ void publish_state(const float (&S)[SD], uint8_t *at, int lane) {
#pragma unroll
  for (int c = 0; c < 16; c++) {
    uint4 x;
    x.x = pack_bf16(S[8 * c], S[8 * c + 1]);
    x.y = pack_bf16(S[8 * c + 2], S[8 * c + 3]);
    x.z = pack_bf16(S[8 * c + 4], S[8 * c + 5]);
    x.w = pack_bf16(S[8 * c + 6], S[8 * c + 7]);
    *reinterpret_cast<uint4 *>(at + (c / 8) * HALF + (((c % 8) ^ (lane & 7)) << 4)) = x;
  }
}

// What a lane has of a block's gates before they are worked out: four consecutive rows of beta (or dt) and alpha.
template <typename G, bool SELECT>
struct RawGates {
  G beta[4], alpha[4];
  int rows;                                    // rows of the block
  int h;
  __device__ __forceinline__ void load(const ScanArgs &a, int row, int rows_, int h_, int lane) {
    rows = rows_, h = h_;
    const G *b = static_cast<const G *>(a.beta) + h, *al = static_cast<const G *>(a.alpha) + h;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = row + min(4 * lane + i, rows - 1);       // (rows that are not there: loaded from the last one that is)
      beta[i] = b[r * a.beta_stride];
      if (!SELECT) alpha[i] = al[r * a.alpha_stride];
    }
  }
};

// A lane's part of the block's gates, four consecutive rows: worked out, then written when there is room.
struct LaneGates {
  float4 minus_whole, minus_frac, beta, e;
  float end_whole, end_frac, rest, total;
};
template <typename G, bool SELECT>
__device__ __forceinline__ LaneGates scan_gates(const ScanArgs &a, const RawGates<G, SELECT> &raw, int lane) {
  float whole[4], frac[4], beta[4];
  float sw = 0.0f, sf = 0.0f;
  const float bias = SELECT && a.dt_bias ? a.dt_bias[raw.h] : 0.0f, rate = SELECT ? a.A[raw.h] * 1.44269504088896340736f : 0.0f;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const bool there = 4 * lane + i < raw.rows;
    float b = to_float(raw.beta[i]), l;
    if (SELECT) {
      b = softplus(b + bias);
      l = b * rate;
    } else {
      l = log2f(to_float(raw.alpha[i]));
    }
    if (l < -200.0f) l = -200.0f;              // (2^-200 is 0 in binary32; a NaN stays)
    b = there ? b : 0.0f;
    l = there ? l : 0.0f;
    beta[i] = b;
    const float r = rintf(l);
    sw += r;
    sf += l - r;
    whole[i] = sw;
    frac[i] = sf;
  }
  float uw = sw, uf = sf;                      // sums over the lanes up to this one
#pragma unroll
  for (int m = 1; m < 32; m *= 2) {
    const float w = __shfl_up_sync(0xffffffffu, uw, m), f = __shfl_up_sync(0xffffffffu, uf, m);
    if (lane >= m) uw += w, uf += f;
  }
  const int ender = lane | 7;                  // the lane that ends these 32 rows
  const float rw = __shfl_sync(0xffffffffu, uw, ender), rf = __shfl_sync(0xffffffffu, uf, ender);
  const float tw = __shfl_sync(0xffffffffu, uw, 31), tf = __shfl_sync(0xffffffffu, uf, 31);
  uw -= sw;
  float before = __shfl_up_sync(0xffffffffu, uf, 1);
  if (lane == 0) before = 0.0f;
  LaneGates g;
  g.end_whole = rw, g.end_frac = rf, g.rest = exp2_fast((tw - rw) + (tf - rf)), g.total = exp2_fast(tw + tf);
  g.beta = make_float4(beta[0], beta[1], beta[2], beta[3]);
  float *pw = &g.minus_whole.x, *pf = &g.minus_frac.x, *pe = &g.e.x;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float w = uw + whole[i], f = before + frac[i];
    pw[i] = -w;
    pf[i] = -f;
    pe[i] = beta[i] * exp2_fast((rw - w) + (rf - f));
  }
  return g;
}

// Values of 16 rows and 16 channels times the rows' weights, in three bf16 pieces: the leading 8 bits, the next 8, the rest - together all 24.
// `at`: this lane's address for four transposed 8 x 8 matrices; afterwards the lane has two rows (weights w[m / 2]) of one channel in each.
__device__ __forceinline__ void weigh_values(uint32_t at, const float2 (&w)[2], uint32_t (&hi)[4], uint32_t (&mid)[4], uint32_t (&low)[4]) {
  uint32_t v[4];
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
  const float2 minus = make_float2(-1.0f, -1.0f);
  auto top = [](float2 x) { return make_float2(__uint_as_float(__float_as_uint(x.x) & 0xFFFF0000u), __uint_as_float(__float_as_uint(x.y) & 0xFFFF0000u)); };
  auto tops = [](float2 x) { return __byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x7632); };
#pragma unroll
  for (int m = 0; m < 4; m++) {
    float2 x = __fmul2_rn(w[m / 2], make_float2(__uint_as_float(v[m] << 16), __uint_as_float(v[m] & 0xFFFF0000u)));
    hi[m] = tops(x);
    x = __ffma2_rn(top(x), minus, x);
    mid[m] = tops(x);
    x = __ffma2_rn(top(x), minus, x);
    low[m] = tops(x);
  }
}

// One arrival for a warp whose lanes have all come this far; what they wrote is visible to who waits.
__device__ __forceinline__ void warp_arrive(uint64_t &bar, int lane) {
  __syncwarp();
  if (lane == 0) bar_arrive(shared_addr(&bar));
}

// The CTA's next item; false: a wait ran out.
__device__ __forceinline__ bool take(ScanShared &sm, ScanItem &it, int &t, int lane) {
  if (!wait_for(sm.items_full[t & 1], (t >> 1) & 1)) return false;
  const int *x = sm.items[t & 1];
  it.h = x[0], it.slot = x[1], it.row = x[2], it.rows = x[3], it.at = x[4], it.flags = x[5];
  it.blocks = (it.rows + SB - 1) / SB;
  warp_arrive(sm.items_empty[t & 1], lane);
  t++;
  return true;
}

// ---- warp 0 (one thread): items, tensor copies ----
template <bool OUT>
__device__ __forceinline__ void scan_copies(ScanShared &sm, const ScanMaps &maps, const ScanArgs &a, const ScanPlan &plan) {
  ScanItem it;
  int c = 0, ns = 0, asked[3] = {0, 0, 0};     // blocks; states that they are given; tiles of K, Q, V that have been asked for
  bool ok = true;
  if (a.sq.tokens > 0) {                       // (without rows there are no maps)
    tensor_map_prefetch(&maps.k);
    tensor_map_prefetch(&maps.v);
    if (OUT) tensor_map_prefetch(&maps.q);
  }
  auto copy = [&](const CUtensorMap *map, uint8_t (&to)[2][TILE], int head, int row, uint64_t (&full)[2], uint64_t (&empty)[2], int &count) {
    const int r = c & 1;
    if (c >= 2 && !(ok = wait_one(empty[r], ((c >> 1) + 1) & 1))) return false;
    const uint32_t bar = shared_addr(&full[r]), dst = shared_addr(to[r]);
    bar_expect(bar, TILE);
    tensor_g2s(dst, map, 0, head, row, bar);
    tensor_g2s(dst + HALF, map, 64, head, row, bar);
    count++;
    return true;
  };
  int item = blockIdx.x, behind = 0;
  for (int t = 0; ok; t++) {
    bool found = false;
    for (; item < plan.items && !found; item = behind) {
      behind = plan.next ? (int)gridDim.x + atomicAdd(plan.next, 1) : item + (int)gridDim.x;   // (needed at the end of this item)
      found = it.find<OUT>(a, plan, item);
    }
    if (t >= 2 && !(ok = wait_one(sm.items_empty[t & 1], ((t >> 1) + 1) & 1))) break;
    int *x = sm.items[t & 1];
    x[0] = it.h, x[1] = it.slot, x[2] = it.row, x[3] = found ? it.rows : -1, x[4] = it.at, x[5] = it.flags;
    bar_arrive(shared_addr(&sm.items_full[t & 1]));
    if (!found) break;
    const int hq = plan.group.quotient(it.h);
    for (int row = it.row; row < it.row + it.rows; row += SB, c++) {
      if (OUT && !copy(&maps.q, sm.q, hq, row, sm.q_full, sm.q_empty, asked[1])) break;   // (Q is through first)
      if (!copy(&maps.k, sm.k, hq, row, sm.k_full, sm.k_empty, asked[0])) break;
      if (!copy(&maps.v, sm.v, it.h, row, sm.v_full, sm.v_empty, asked[2])) break;
      ns += OUT && (it.state() || row > it.row);
    }
  }
  if (ok && c > 0) {                           // the products' arrivals that nobody waits for any more, before their barriers are gone: in the order in which they come
    for (int i = max(c - 2, 0); ok && i < c; i++) {
      const int r = i & 1, parity = (i >> 1) & 1;
      ok = (!OUT || wait_one(sm.q_empty[r], parity)) && wait_one(sm.k_empty[r], parity);
      // (behind those: of the phase before have all been waited for, or the last block's products would not have been issued)
      if (i == c - 1) ok = ok && (ns == 0 || wait_one(sm.s_empty, (ns + 1) & 1)) && wait_one(sm.w_empty[0], 1) && wait_one(sm.w_empty[1], 1);
      ok = ok && wait_one(sm.v_empty[r], parity);
    }
    if (!ok) atomicOr(&g_ops_error, 1);
  } else if (!ok) {                            // the copies that nobody waited for: the last two of each kind
    atomicOr(&g_ops_error, 1);
    auto landed = [](uint64_t (&full)[2], int n) {
      for (int i = max(n - 2, 0); i < n; i++)
        for (int spin = 0; spin < WAIT_LIMIT && !bar_try(shared_addr(&full[i & 1]), (i >> 1) & 1); spin++) {
        }
    };
    landed(sm.k_full, asked[0]);
    landed(sm.q_full, asked[1]);
    landed(sm.v_full, asked[2]);
  }
}

__device__ __forceinline__ void gave_up(bool yes) {
  if (yes) atomicOr(&g_ops_error, 1);
}

// What a warp of matrix instructions does in the end where somebody gave up: what it has under way ends before tensor memory is freed.
__device__ __forceinline__ void drain(uint64_t &bar) {
  if (elect_one()) {
    mma_commit(shared_addr(&bar));
    for (int spin = 0; spin < WAIT_LIMIT && !bar_try(shared_addr(&bar), 0); spin++) {
    }
  }
  __syncwarp();
}

// A product over 128 channels, two halves of 64 that lie HALF apart, anew.
__device__ __forceinline__ void multiply_halves(uint32_t d, Operand a, Operand b, uint32_t what) {
#pragma unroll 1
  for (int half = 0; half < 2; half++) {
    mma_ss(d, a + half * HALF, b + half * HALF, what, half > 0);
#pragma unroll
    for (int s = 1; s < 4; s++) mma_ss<true>(d, a + (half * HALF + s * 32), b + (half * HALF + s * 32), what);
  }
}

// ---- warp 1: the products for the outputs ----
__device__ __forceinline__ void scan_products(ScanShared &sm, int lane) {
  constexpr uint32_t KK = mma_bf16(128, 128, false, false), KN = mma_bf16(128, 128, false, true);
  const Operand S = operand(shared_addr(sm.s16), 16, 1024);
  ScanItem it;
  int t = 0, c = 0, ns = 0;                    // items, blocks, states published so far
  bool ok = true;
  while (ok && (ok = take(sm, it, t, lane)) && it.rows >= 0) {
    for (int b = 0; b < it.blocks; b++, c++) {
      const int r = c & 1;
      if (!(ok = wait_for(sm.k_full[r], (c >> 1) & 1))) break;
      if (!(ok = wait_for(sm.q_full[r], (c >> 1) & 1))) break;
      if (c > 0 && !(ok = wait_for(sm.o_full, (c + 1) & 1))) break;   // (the product that reads the weighted P of the block before)
      tmem_fence_after();
      const Operand K = operand(shared_addr(sm.k[0]) + r * TILE, 16, 1024), Q = operand(shared_addr(sm.q[0]) + r * TILE, 16, 1024), V = operand(shared_addr(sm.v[0]) + r * TILE, HALF, 1024);
      if (elect_one()) {                       // P = Q K^T
        multiply_halves(TM_P, Q, K, KK);
        mma_commit(shared_addr(&sm.p_full));
        mma_commit(shared_addr(&sm.k_empty[r]));
      }
      __syncwarp();
      const bool state = it.state() || b > 0;
      if (c > 0 && !(ok = wait_for(sm.o_free, (c + 1) & 1))) break;
      if (state) {                             // O = Q S
        if (!(ok = wait_for(sm.s_full, ns++ & 1))) break;
        tmem_fence_after();
        if (elect_one()) {
          multiply_halves(TM_O, Q, S, KK);
          mma_commit(shared_addr(&sm.s_empty));
        }
        __syncwarp();
      }
      if (elect_one()) mma_commit(shared_addr(&sm.q_empty[r]));
      __syncwarp();
      if (!(ok = wait_for(sm.v_full[r], (c >> 1) & 1))) break;
      if (!(ok = wait_for(sm.clean[r], (c >> 1) & 1))) break;
      if (!(ok = wait_for(sm.pw_full, c & 1))) break;
      tmem_fence_after();
      if (elect_one()) {                       // O += (weighted P) V
#pragma unroll 2
        for (int s = 0; s < 8; s++) mma_ts(TM_O, TM_P + 8 * s, V + s * 2048, KN, state || s > 0);
        mma_commit(shared_addr(&sm.o_full));
        mma_commit(shared_addr(&sm.v_empty[r]));
      }
      __syncwarp();
    }
  }
  if (!ok) drain(sm.drained[0]);
  gave_up(!ok);
}

// ---- warp 3: the product for the state, dS^T = (weighted V)^T K, the small pieces first ----
__device__ __forceinline__ void scan_state_product(ScanShared &sm, int lane) {
  constexpr uint32_t KN = mma_bf16(128, 128, false, true);
  ScanItem it;
  int t = 0, c = 0;
  bool ok = true;
  while (ok && (ok = take(sm, it, t, lane)) && it.rows >= 0) {
    for (int b = 0; b < it.blocks; b++, c++) {
      const int r = c & 1;
      if (!(ok = wait_for(sm.k_full[r], (c >> 1) & 1))) break;
      if (c > 0 && !(ok = wait_for(sm.ds_free, (c + 1) & 1))) break;
      const Operand K = operand(shared_addr(sm.k[0]) + r * TILE, HALF, 1024);
#pragma unroll 1
      for (int q = 0; q < SB / 32; q++) {
        const int u = q & 1;
        if (!(ok = wait_for(sm.w_full[u], q >> 1))) break;   // (two uses of a buffer in a block)
        tmem_fence_after();
        const uint32_t W = TM_W + 48 * u;
        const Operand y = K + q * 4096;
        if (elect_one()) {
          mma_ts(TM_DS, W + 16, y, KN, q > 0);
          mma_ts<true>(TM_DS, W + 8, y, KN);
          mma_ts<true>(TM_DS, W, y, KN);
          mma_ts<true>(TM_DS, W + 40, y + 2048, KN);
          mma_ts<true>(TM_DS, W + 32, y + 2048, KN);
          mma_ts<true>(TM_DS, W + 24, y + 2048, KN);
          mma_commit(shared_addr(&sm.w_empty[u]));
        }
        __syncwarp();
      }
      if (!ok) break;
      if (elect_one()) {
        mma_commit(shared_addr(&sm.ds_full));
        mma_commit(shared_addr(&sm.k_empty[r]));
        mma_commit(shared_addr(&sm.v_empty[r]));
      }
      __syncwarp();
    }
  }
  if (!ok) drain(sm.drained[1]);
  gave_up(!ok);
}

// ---- warps 4 - 7: weights on P.  A thread has row i = 32 w + lane ----
__device__ __forceinline__ void scan_weights(ScanShared &sm, int w, int lane) {
  const int i = 32 * w + lane;
  const uint32_t mine = ((uint32_t)(32 * w) << 16);
  ScanItem it;
  int t = 0, c = 0;
  bool ok = true;
  while (ok && (ok = take(sm, it, t, lane)) && it.rows >= 0) {
    for (int b = 0; b < it.blocks; b++, c++) {
      const ScanWeights &g = sm.weights[c & 1];
      const int rows = min(it.rows - b * SB, SB);
      if (!(ok = wait_for(sm.sums_full, c & 1))) break;      // (the weights are there before the sums)
      const bool far = -sm.sums.minus_whole[i] < LEAST;      // (of G_i, what is not in the output's factor)
      const float whole = far ? -sm.sums.minus_whole[i] - LEAST : 0.0f, frac = far ? -sm.sums.minus_frac[i] : 0.0f;
      if (!(ok = wait_for(sm.p_full, c & 1))) break;
      tmem_fence_after();
#pragma unroll 1
      for (int col = 0; col < 32 * (w + 1); col += 16) {
        uint32_t p[16], packed[8];
        tmem_load16(mine + TM_P + col, p);
        const int group = col / 32;
        float2 x[8];
        if (group < w) {                       // all rows below these columns: exp(G_i - G_end) exp(G_end - G_j), the second at most 1
          const float f = exp2_fast((whole - g.end_whole[group]) + (frac - g.end_frac[group]));
#pragma unroll
          for (int j = 0; j < 8; j++) x[j] = __fmul2_rn(make_float2(f, f), *reinterpret_cast<const float2 *>(g.e + col + 2 * j));
        } else {
          const int last = min(i, rows - 1) - col;   // (columns of rows that are not there: nothing, whatever P holds)
#pragma unroll
          for (int j = 0; j < 8; j++) {
            const float2 d = __fadd2_rn(__fadd2_rn(make_float2(whole, whole), *reinterpret_cast<const float2 *>(sm.sums.minus_whole + col + 2 * j)),
                                        __fadd2_rn(make_float2(frac, frac), *reinterpret_cast<const float2 *>(sm.sums.minus_frac + col + 2 * j)));
            x[j] = __fmul2_rn(*reinterpret_cast<const float2 *>(sm.sums.beta + col + 2 * j), make_float2(exp2_fast(d.x), exp2_fast(d.y)));
          }
          tmem_wait_loads(p);
#pragma unroll
          for (int j = 0; j < 16; j++) p[j] = j <= last ? p[j] : 0;
#pragma unroll
          for (int j = 0; j < 8; j++) x[j] = make_float2(2 * j <= last ? x[j].x : 0.0f, 2 * j + 1 <= last ? x[j].y : 0.0f);
        }
        tmem_wait_loads(p);
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const float2 y = __fmul2_rn(x[j], make_float2(__uint_as_float(p[2 * j]), __uint_as_float(p[2 * j + 1])));
          packed[j] = pack_bf16(y.x, y.y);
        }
        tmem_store8(mine + TM_P + col / 2, packed);
      }
#pragma unroll 1
      for (int col = w + 1; col < 4; col++) {  // above the diagonal there is nothing
        uint32_t zero[16];
#pragma unroll
        for (int j = 0; j < 16; j++) zero[j] = 0;
        tmem_store16(mine + TM_P + 16 * col, zero);
      }
      tmem_wait_stores();
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) {
        bar_arrive(shared_addr(&sm.pw_full));
        bar_arrive(shared_addr(&sm.sums_empty));
        bar_arrive(shared_addr(&sm.weights_empty[c & 1]));
      }
    }
  }
  gave_up(!ok);
}

__device__ __forceinline__ void store_sector(void *to, const uint32_t (&x)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]),
               "r"(x[6]), "r"(x[7])
               : "memory");
}

// ---- warps 8 - 15: outputs.  A thread has row i = 32 w + lane and columns 64 * half .. 64 * half + 63 ----
__device__ __forceinline__ void scan_outputs(ScanShared &sm, const ScanArgs &a, int warp, int lane) {
  const int half = warp / 4, w = warp % 4, i = 32 * w + lane;
  const uint32_t mine = ((uint32_t)(32 * w) << 16) + TM_O + 64 * half;
  const bool sectors = reinterpret_cast<uintptr_t>(a.o) % 32 == 0 && a.o_stride % 16 == 0;   // a row's pieces are whole 32-byte sectors
  ScanItem it;
  int t = 0, c = 0;
  bool ok = true;
  while (ok && (ok = take(sm, it, t, lane)) && it.rows >= 0) {
    const float skip = a.skip ? a.skip[it.h] : 0.0f;
    __nv_bfloat16 *out = static_cast<__nv_bfloat16 *>(a.o) + (int64_t)(it.row + i) * a.o_stride + it.h * SD + 64 * half;
    for (int b = 0; b < it.blocks; b++, c++) {
      if (!(ok = wait_for(sm.sums_full, c & 1))) break;
      const float whole = -sm.sums.minus_whole[i], g = exp2_fast(whole >= LEAST ? whole - sm.sums.minus_frac[i] : LEAST);
      const float2 gamma = make_float2(g, g);
      warp_arrive(sm.sums_empty, lane);
      if (!(ok = wait_for(sm.v_full[c & 1], (c >> 1) & 1))) break;
      if (!(ok = wait_for(sm.o_full, c & 1))) break;
      tmem_fence_after();
      const bool there = it.row + b * SB + i < it.row + it.rows;
      const uint8_t *V = sm.v[c & 1] + half * HALF + i * 128;
#pragma unroll 1
      for (int col = 0; col < 4; col++) {
        uint32_t o[16], y[8];
        tmem_load16(mine + 16 * col, o);
        uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        if (a.skip) {
          x[0] = *reinterpret_cast<const uint4 *>(V + (((2 * col) ^ (i & 7)) << 4));
          x[1] = *reinterpret_cast<const uint4 *>(V + (((2 * col + 1) ^ (i & 7)) << 4));
        }
        const uint32_t in[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
        tmem_wait_loads(o);
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const float2 v = __fmul2_rn(make_float2(skip, skip), make_float2(__uint_as_float(in[j] << 16), __uint_as_float(in[j] & 0xFFFF0000u)));
          const float2 z = __ffma2_rn(gamma, make_float2(__uint_as_float(o[2 * j]), __uint_as_float(o[2 * j + 1])), v);
          y[j] = pack_bf16(z.x, z.y);
        }
        if (there) {                           // a thread's 32 bytes of a row: one sector where the rows allow it
          if (sectors) {
            store_sector(out + 16 * col, y);
          } else {
            reinterpret_cast<uint4 *>(out + 16 * col)[0] = make_uint4(y[0], y[1], y[2], y[3]);
            reinterpret_cast<uint4 *>(out + 16 * col)[1] = make_uint4(y[4], y[5], y[6], y[7]);
          }
        }
      }
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) {
        bar_arrive(shared_addr(&sm.o_free));
        bar_arrive(shared_addr(&sm.v_empty[c & 1]));
      }
      out += SB * a.o_stride;
    }
  }
  gave_up(!ok);
}

// ---- warps 16 - 23: weighted values.  A warp has value channels 32 w .. 32 w + 31, the warps of a half have every other 16 rows ----
__device__ __forceinline__ void scan_values(ScanShared &sm, int warp, int lane) {
  const int half = warp / 4, w = warp % 4, thread = 32 * warp + lane;
  const uint32_t mine = ((uint32_t)(32 * w) << 16) + TM_W + 24 * half;
  // matrix lane / 8: channels 8 (lane / 8 % 2) of 16, rows 8 (lane / 16) of 16
  const int mrow = 8 * (lane / 16) + lane % 8, chunk = 4 * (w & 1) + (lane / 8) % 2;
  const uint32_t first = (w >> 1) * HALF + half * 2048 + mrow * 128, pick[2] = {(uint32_t)((chunk ^ (lane % 8)) << 4), (uint32_t)(((chunk + 2) ^ (lane % 8)) << 4)};
  ScanItem it;
  int t = 0, c = 0;
  bool ok = true;
  while (ok && (ok = take(sm, it, t, lane)) && it.rows >= 0) {
    for (int b = 0; b < it.blocks; b++, c++) {
      const int rows = min(it.rows - b * SB, SB);
      uint8_t *V = sm.v[c & 1];
      if (!(ok = wait_for(sm.weights_full[c & 1], (c >> 1) & 1))) break;
      if (!(ok = wait_for(sm.v_full[c & 1], (c >> 1) & 1))) break;
      if (rows < SB) {                         // rows of another sequence, or of none: what they hold must not meet the weights 0
        if (!(ok = wait_for(sm.k_full[c & 1], (c >> 1) & 1))) break;
        uint8_t *K = sm.k[c & 1];
        for (int u = thread; u < (SB - rows) * 16; u += 256) {
          const uint32_t off = (u & 1) * HALF + rows * 128 + (u >> 1) * 16;
          *reinterpret_cast<uint4 *>(K + off) = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4 *>(V + off) = make_uint4(0, 0, 0, 0);
        }
        fence_async_shared();
      }
      warp_arrive(sm.clean[c & 1], lane);
      if (rows < SB && !(ok = wait_for(sm.clean[c & 1], (c >> 1) & 1))) break;
      const uint32_t v = shared_addr(V) + first;
      const ScanWeights &g = sm.weights[c & 1];
      const float *weights = g.e + 16 * half + 2 * (lane % 4);
#pragma unroll 1
      for (int q = 0; q < SB / 32; q++) {
        uint32_t hi[2][4], mid[2][4], low[2][4];
        const float2 rest = make_float2(g.rest[q], g.rest[q]);
        const float2 x[2] = {__fmul2_rn(rest, *reinterpret_cast<const float2 *>(weights + 32 * q)),
                             __fmul2_rn(rest, *reinterpret_cast<const float2 *>(weights + 32 * q + 8))};
#pragma unroll
        for (int i = 0; i < 2; i++) weigh_values(v + q * 4096 + pick[i], x, hi[i], mid[i], low[i]);
        const int u = q & 1;                   // two uses of a buffer in a block
        if ((c > 0 || q > 1) && !(ok = wait_for(sm.w_empty[u], (q >> 1) ^ 1))) break;
        tmem_fence_after();
#pragma unroll
        for (int i = 0; i < 2; i++) {
          const uint32_t lanes = mine + 48 * u + ((uint32_t)(16 * i) << 16);
          tmem_store_16x8(lanes, hi[i]);
          tmem_store_16x8(lanes + 8, mid[i]);
          tmem_store_16x8(lanes + 16, low[i]);
        }
        tmem_wait_stores();
        tmem_fence_before();
        warp_arrive(sm.w_full[u], lane);
      }
      if (!ok) break;
      warp_arrive(sm.weights_empty[c & 1], lane);
    }
  }
  gave_up(!ok);
}

// ---- warps 24 - 27: the state.  A thread has value channel 32 w + lane ----
template <bool OUT>
__device__ __forceinline__ void scan_state(ScanShared &sm, const ScanArgs &a, const ScanPlan &plan, int w, int lane) {
  const uint32_t mine = ((uint32_t)(32 * w) << 16) + TM_DS;
  const int channel = 32 * w + lane;
  uint8_t *s16 = sm.s16 + channel * 128;
  ScanItem it;
  int t = 0, c = 0, ns = 0;                    // items, blocks, states published so far
  bool ok = true;
  while (ok && (ok = take(sm, it, t, lane)) && it.rows >= 0) {
    const size_t at = it.at;
    const size_t slot = ((size_t)it.slot * a.heads_v + it.h) * (SD * SD) + channel;
    const bool keep = it.state() && it.blocks == 0 && a.S0 == a.S;   // no rows: the state is where it belongs
    float S[SD];
#pragma unroll
    for (int j = 0; j < SD; j++) S[j] = 0.0f;
    if (it.state() && !keep) load_state(S, plan.pieces > 1 ? plan.states + at * (SD * SD) + channel : a.S0 + slot);
    float decay = 1.0f;
    for (int b = 0; b < it.blocks; b++, c++) {
      if (OUT && (it.state() || b > 0)) {
        // The product that reads the state published last.  (One phase for every state, not for every block: fresh heads' first blocks have none,
        // and a wait that they leave out would find a phase of blocks one behind and take it for the one after.)
        if (ns > 0 && !(ok = wait_for(sm.s_empty, (ns + 1) & 1))) break;
        ns++;
        publish_state(S, s16, lane);
        fence_async_shared();
        warp_arrive(sm.s_full, lane);
      }
      if (!(ok = wait_for(sm.weights_full[c & 1], (c >> 1) & 1))) break;
      const float gamma = sm.weights[c & 1].total;
      warp_arrive(sm.weights_empty[c & 1], lane);
      decay *= gamma;
      if (!(ok = wait_for(sm.ds_full, c & 1))) break;
      tmem_fence_after();
#pragma unroll
      for (int col = 0; col < 8; col++) {
        uint32_t d[16];
        tmem_load16(mine + 16 * col, d);
        tmem_wait_loads(d);
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          const float2 x = __ffma2_rn(make_float2(gamma, gamma), make_float2(S[16 * col + j], S[16 * col + j + 1]),
                                      make_float2(__uint_as_float(d[j]), __uint_as_float(d[j + 1])));
          S[16 * col + j] = x.x;
          S[16 * col + j + 1] = x.y;
        }
      }
      tmem_fence_before();
      warp_arrive(sm.ds_free, lane);
    }
    if (!ok) break;
    if (OUT) {
      if (it.last() && !keep) store_state(S, a.S + slot);
    } else {
      store_state(S, plan.states + (at + a.heads_v) * (SD * SD) + channel);
      if (channel == 0) plan.decays[at] = decay;
    }
  }
  gave_up(!ok);
}

// ---- warp 2: gates.  The next block's are loaded before this block's are worked out ----
template <bool OUT, typename G, bool SELECT>
__device__ __forceinline__ void scan_gate_warp(ScanShared &sm, const ScanArgs &a, int lane) {
  ScanItem it;
  RawGates<G, SELECT> next;
  int t = 0, b = 0, c = 0;
  bool more = false, over = false, ok = true;
  it.blocks = 0;
  while (more || !over) {
    const RawGates<G, SELECT> now = next;
    const bool have = more;
    // One item ahead at most: the one behind it is not handed out before everybody has taken this one, for which they wait for these gates.
    if (!over && b >= it.blocks) {
      if (!(ok = take(sm, it, t, lane))) break;
      over = it.rows < 0;
      b = 0;
    }
    more = !over && b < it.blocks;
    if (more) {
      next.load(a, it.row + b * SB, min(it.rows - b * SB, SB), it.h, lane);
      b++;
    }
    if (!have) continue;
    const LaneGates g = scan_gates(a, now, lane);
    if (c >= 2 && !(ok = wait_for(sm.weights_empty[c & 1], ((c >> 1) + 1) & 1))) break;
    ScanWeights &w = sm.weights[c & 1];
    reinterpret_cast<float4 *>(w.e)[lane] = g.e;
    if (lane % 8 == 7) w.end_whole[lane / 8] = g.end_whole, w.end_frac[lane / 8] = g.end_frac, w.rest[lane / 8] = g.rest;
    if (lane == 0) w.total = g.total;
    warp_arrive(sm.weights_full[c & 1], lane);
    if (OUT) {
      if (c >= 1 && !(ok = wait_for(sm.sums_empty, (c + 1) & 1))) break;
      reinterpret_cast<float4 *>(sm.sums.minus_whole)[lane] = g.minus_whole;
      reinterpret_cast<float4 *>(sm.sums.minus_frac)[lane] = g.minus_frac;
      reinterpret_cast<float4 *>(sm.sums.beta)[lane] = g.beta;
      warp_arrive(sm.sums_full, lane);
    }
    c++;
  }
  gave_up(!ok);
}

template <bool OUT, typename G, bool SELECT>
__global__ void __launch_bounds__(SCAN_THREADS, 1) scan_blocks_kernel(const __grid_constant__ ScanMaps maps, const ScanArgs a, const ScanPlan plan) {
  extern __shared__ __align__(1024) uint8_t raw[];
  ScanShared &sm = *reinterpret_cast<ScanShared *>(raw);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (shared_addr(raw) % 1024 != 0) {          // (the swizzled tiles count on it)
    if (threadIdx.x == 0) atomicOr(&g_ops_error, 2);
    return;
  }
  if (threadIdx.x == 0) {
    auto init = [](uint64_t &bar, int count) { bar_init(shared_addr(&bar), count); };
    for (int i = 0; i < 2; i++) {              // K is left by two products, V by two products and the eight warps that add the skip
      init(sm.items_full[i], 1), init(sm.items_empty[i], OUT ? 27 : 14);   // (every warp with a part but the first)
      init(sm.k_full[i], 1), init(sm.k_empty[i], OUT ? 2 : 1), init(sm.q_full[i], 1), init(sm.q_empty[i], 1);
      init(sm.v_full[i], 1), init(sm.v_empty[i], OUT ? 10 : 1);
      init(sm.weights_full[i], 1), init(sm.weights_empty[i], OUT ? 16 : 12);
      init(sm.w_full[i], 8), init(sm.w_empty[i], 1);
      init(sm.clean[i], 8), init(sm.drained[i], 1);
    }
    for (uint64_t *b : {&sm.sums_full, &sm.p_full, &sm.s_empty, &sm.o_full, &sm.ds_full}) init(*b, 1);
    for (uint64_t *b : {&sm.pw_full, &sm.ds_free, &sm.s_full}) init(*b, 4);
    init(sm.o_free, 8);
    init(sm.sums_empty, 12);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 3) tmem_alloc(shared_addr(&sm.tmem), 512);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (sm.tmem != 0) {                          // (all of tensor memory is this CTA's, so its columns start at 0: the addresses are constants)
    if (threadIdx.x == 0) atomicOr(&g_ops_error, 2);
    __syncthreads();
    if (warp == 3) tmem_free(sm.tmem, 512);
    return;
  }
  // 896 threads start with 72 registers each, 64512 in all: dealt out anew, 128 * (56 + 72 + 168) + 256 * (48 + 56)
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0) {
      if (lane == 0) scan_copies<OUT>(sm, maps, a, plan);
    } else if (warp == 1) {
      if (OUT) scan_products(sm, lane);
    } else if (warp == 2) {
      scan_gate_warp<OUT, G, SELECT>(sm, a, lane);
    } else {
      scan_state_product(sm, lane);
    }
  } else if (warp < 8) {
    if (OUT) scan_weights(sm, warp - 4, lane);
  } else if (warp < 16) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (OUT) scan_outputs(sm, a, warp - 8, lane);
  } else if (warp < 24) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    scan_values(sm, warp - 16, lane);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    scan_state<OUT>(sm, a, plan, warp - 24, lane);
  }
  __syncwarp();
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (warp == 3) tmem_free(0, 512);
}

// In front of a pass with more heads than CTAs (one CTA): the count of those taken is 0, and the sequences by length.  A long prompt that is
// begun last ends long after everything else.
__global__ void __launch_bounds__(1024) scan_order_kernel(const ScanArgs a, const ScanPlan plan) {
  if (threadIdx.x == 0) *plan.next = 0;
  __shared__ int len[4096];
  for (int n = threadIdx.x; n < a.sq.seqs; n += 1024) len[n] = a.sq.slot(n) < 0 ? -1 : min(max(a.sq.first(n + 1) - a.sq.first(n), 0), a.max_len);
  __syncthreads();
  for (int n = threadIdx.x; n < a.sq.seqs; n += 1024) {
    const int mine = len[n];
    int before = 0;
    for (int m = 0; m < a.sq.seqs; m++) before += len[m] > mine || (len[m] == mine && m < n);
    plan.order[before] = n;
  }
}

// From every piece's own sum (in the place of the state in front of the next piece) to the states in front of the pieces.
__global__ void __launch_bounds__(256) scan_join_kernel(const ScanArgs a, const ScanPlan plan) {
  const int r = blockIdx.x / 16, n = r / a.heads_v, h = r - n * a.heads_v;
  const int slot = a.sq.slot(n), start = a.sq.first(n), len = min(max(a.sq.first(n + 1) - start, 0), a.max_len);
  if (slot < 0) return;
  const size_t e = (size_t)(blockIdx.x % 16) * 1024 + threadIdx.x * 4;
  float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (a.sq.resumed(n)) x = *reinterpret_cast<const float4 *>(a.S0 + ((size_t)slot * a.heads_v + h) * (SD * SD) + e);
  for (int p = 0;; p++) {
    const size_t at = ((size_t)n * plan.pieces + p) * a.heads_v + h;
    *reinterpret_cast<float4 *>(plan.states + at * (SD * SD) + e) = x;
    if ((p + 1) * plan.piece >= len) break;
    const float d = plan.decays[at];
    const float4 y = *reinterpret_cast<const float4 *>(plan.states + (at + a.heads_v) * (SD * SD) + e);
    x = make_float4(fmaf(d, x.x, y.x), fmaf(d, x.y, y.y), fmaf(d, x.z, y.z), fmaf(d, x.w, y.w));
  }
}

}  // namespace lq
