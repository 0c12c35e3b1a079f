// Products of e4m3 rows with e4m3 weights, scales for each 128 channels of a row and for each block of 128 x 128 of the weights:
//     out[t][n] = sum_b xs[b][t] ws[n / 128][b] sum_{k in block b} x[t][k] w[n][k]
//
// The inner sums are tcgen05 products (kind::f8f6f4) of one K block, 128 channels, in tensor memory.  Its accumulator is binary32, but an instruction cuts off what is 2^-25
// below the largest of its 32 products and the sum so far: a block is off by 0.5 of 2^-23 of the sum over magnitudes where the products are of one size, by 4 where the
// codes are of every size, by 33 * 2^-25 + 2^-23 four times, 37 of 2^-23, at most.  The outer sum is taken in registers: every K block is read out of tensor memory and
// added with one multiply-add an element, its factor xs ws.  So unlike a product without scales each K block is handed over twice, and that is what bounds the
// large ones: see the kernel for many rows.  Nothing is kept between calls and there is no workspace.
// Both kernels are programmatic dependents and let theirs come up at once, where room appears: one row of 4096 x 4096 8.0 -> 7.3 us, 64 rows 10.9 -> 9.8.
#pragma once
#include "lq_dependent.cuh"
#include "lq_rows.cuh"
#include "lq_tensor.cuh"

namespace lq {

constexpr int PB = 128;                        // channels (and outputs) of a scale; a K block
constexpr int MOST_GROUPS = LQ_MOST_GROUPS;

__device__ int g_product_error = 0;
constexpr int PRODUCT_WAIT_LIMIT = 1 << 20;    // tries of a wait

// Bounded wait; false: it ran out, leave (everybody else's next wait will too).
// (The first try stands by itself: a wait that is over takes 53 clocks, by way of the loop 100.)
__device__ __forceinline__ bool reached(uint32_t bar, uint32_t parity) {
  if (bar_try(bar, parity)) return true;
  int left = PRODUCT_WAIT_LIMIT;
#pragma unroll 1
  while (!bar_try(bar, parity))
    if (--left == 0) return false;
  return true;
}

// The same for warps whose lanes have to stay together: no lane leaves, it goes on with waits of one try each and says so in the end.  (A vote behind every wait
// and what hangs on it made a K block of a product 15 % longer.)
struct Patience {
  int limit = PRODUCT_WAIT_LIMIT;
  __device__ __forceinline__ void wait(uint32_t bar, uint32_t parity) {
    if (!bar_try(bar, parity)) {
      int left = limit;
#pragma unroll 1
      while (!bar_try(bar, parity))
        if (--left <= 0) {
          limit = 1;
          break;
        }
    }
    __syncwarp();
  }
  __device__ __forceinline__ bool gone() const { return __any_sync(0xffffffffu, limit == 1); }
};

struct ProductMaps {
  CUtensorMap x, w, more;                      // more: x in copies of FEW_BOX rows, or what is written
};
struct ProductArgs {
  const float *x_scale, *w_scale;
  void *out;
  int64_t x_scale_stride, out_stride;
  const int32_t *group_start;                  // null: one group of all rows
  int rows, blocks, outs, groups;              // blocks: K blocks; outs: output channels
  int tiles_n;                                 // tiles of output channels
  int split, share, more;                      // few rows: CTAs of a cluster that share a tile's K blocks, `share` each and one more to the first `more`
  Divisor tiles_m;                             // without groups: division by the tiles of rows
};

// The tiles of all groups: a group's tiles of rows, for one tile of output channels after another (those that run at the same time have
// their weights in common).  What group_start holds is brought into [0, rows] and into order here: nothing outside of the arrays is
// touched whatever it holds.
struct GroupTiles {
  int first[MOST_GROUPS + 1];                  // tiles of rows in front of a group
  int start[MOST_GROUPS + 1];

  // all threads of the CTA; T: rows of a tile
  __device__ __forceinline__ void find(const ProductArgs &a, int T) {
    if (a.group_start) {
      for (int g = threadIdx.x; g <= a.groups; g += blockDim.x) start[g] = min(max(a.group_start[g], 0), a.rows);
      __syncthreads();
      scan(a, T);
    }
    __syncthreads();
  }
  __device__ __forceinline__ void scan(const ProductArgs &a, int T) {
    if (threadIdx.x < 32) {                    // (running maximum, running sum; 32 groups at a time)
      const int lane = threadIdx.x;
      int high = start[0], sum = 0;
      for (int g0 = 0; g0 < a.groups; g0 += 32) {
        const int g = g0 + lane;
        int s = g < a.groups ? start[g + 1] : 0;
        s = max(s, high);
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
          const int o = __shfl_up_sync(0xffffffffu, s, m);
          if (lane >= m) s = max(s, o);
        }
        int before = __shfl_up_sync(0xffffffffu, s, 1);
        if (lane == 0) before = high;
        const int mine = (s - before + T - 1) / T;
        int n = mine;
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
          const int o = __shfl_up_sync(0xffffffffu, n, m);
          if (lane >= m) n += o;
        }
        __syncwarp();
        if (g < a.groups) start[g + 1] = s, first[g] = sum + n - mine;
        high = __shfl_sync(0xffffffffu, s, 31);
        sum += __shfl_sync(0xffffffffu, n, 31);
      }
      if (lane == 0) first[a.groups] = sum;
    }
  }
};

struct ProductTile {
  int group, row, rows, n;                     // rows [row, row + rows), output channels from n * (channels of a tile) on
  __device__ __forceinline__ bool find(const ProductArgs &a, const GroupTiles &gt, int tile, int T) {
    if (!a.group_start) {
      group = 0, n = a.tiles_m.quotient(tile), row = (tile - n * a.tiles_m.d) * T, rows = min(a.rows - row, T);
      return n < a.tiles_n;
    }
    if (tile >= gt.first[a.groups] * a.tiles_n) return false;
    const int q = tile / a.tiles_n;
    int lo = 0, hi = a.groups;                 // the last group with first <= q
    while (hi - lo > 1) {
      const int m = (lo + hi) / 2;
      if (gt.first[m] <= q) lo = m;
      else hi = m;
    }
    group = lo;
    const int in = tile - gt.first[lo] * a.tiles_n, tiles = gt.first[lo + 1] - gt.first[lo];
    n = in / tiles;
    const int t = in - n * tiles;
    row = gt.start[lo] + t * T;
    rows = min(gt.start[lo + 1] - row, T);
    return true;
  }
};

// ---------------------------------------------------------------------------------------------
// Few rows: output channels are the rows of the accumulator (the lanes of tensor memory), rows of x its columns, as many as there are (in steps of 16).
// The weights are what such a call reads, so all that counts is that they are on their way: 96 KB to an SM, 128 KB with tiles of 32 rows (two CTAs).
// Where there are fewer tiles than SMs, the CTAs of a cluster share a tile's K blocks and add up their sums by way of one another's shared memory, each for
// some of the rows, in the order of the CTAs.  Four accumulators, so that no hand-over is waited for; a K block's factors arrive on the barrier of its sums.
// Weights from memory (not L2): 128 groups of 0 - 100 rows x 2048 x 1536 68 us, 5.9 TB/s; one row of 4096 x 4096 7.1 us, of 4096 x 12352 13.5 us, 3.8 TB/s: 97 CTAs with 64 KB on
// their way each, and 4 us until the first K block is there and after the last.
// ---------------------------------------------------------------------------------------------
constexpr int FEW_THREADS = 384, FEW_ROWS = 128, FEW_BOX = 32;   // FEW_BOX: rows to a copy where there are few
// ROWS: rows of a tile, FEW_ROWS with one CTA to an SM or FEW_BOX with two
template <int ROWS>
struct FewShared {
  static constexpr int STAGES = ROWS == FEW_ROWS ? 6 : 4, SUMS = 4;
  static constexpr uint32_t W_BYTES = PB * PB, BOX_BYTES = FEW_BOX * PB;
  uint8_t w[STAGES][W_BYTES];                  // (behind a split tile's products: sums of all CTAs, [CTA][row][128 channels])
  uint8_t x[STAGES][ROWS * PB];
  uint8_t out[8][16 * 32 * 4];                 // 32 output channels of 16 rows, a warp each
  float factor[2 * SUMS][ROWS];
  uint64_t full[STAGES], empty[STAGES], sum_full[SUMS], sum_empty[SUMS], drained;
  uint32_t tmem;
  GroupTiles tiles;
};

__device__ __forceinline__ void store_shared_of(uint32_t addr, float x) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(x) : "memory"); }

// 32 output channels (a lane each) of 16 rows, of which `rows` and `n` are there, by way of shared memory: pieces of 16 bytes.
template <bool WIDE, typename T>
__device__ __forceinline__ void store_columns(uint8_t *stage, T *dst, int64_t stride, const float *v, int rows, int n, int lane) {
  T *s = reinterpret_cast<T *>(stage);
#pragma unroll
  for (int i = 0; i < 16; i++) s[32 * i + lane] = from_float<T>(v[i]);
  __syncwarp();
  if (WIDE && n >= 32) {
    constexpr int PIECES = 2 * sizeof(T), N = 16 / sizeof(T);   // pieces of a row
#pragma unroll
    for (int u = lane; u < 16 * PIECES; u += 32)
      if (u / PIECES < rows) *reinterpret_cast<uint4 *>(dst + u / PIECES * stride + u % PIECES * N) = reinterpret_cast<const uint4 *>(stage)[u];
  } else if (lane < n) {
#pragma unroll 1
    for (int i = 0; i < rows; i++) dst[i * stride + lane] = s[32 * i + lane];
  }
  __syncwarp();
}

template <typename T, bool WIDE, int ROWS>
__global__ void __launch_bounds__(FEW_THREADS, ROWS == FEW_ROWS ? 1 : 2) product_few_kernel(const __grid_constant__ ProductMaps maps, const ProductArgs a) {
  extern __shared__ __align__(1024) uint8_t raw[];
  using S = FewShared<ROWS>;
  S &sm = *reinterpret_cast<S *>(raw);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (shared_addr(raw) % 1024 != 0) {          // (the swizzled tiles count on it)
    if (threadIdx.x == 0) atomicOr(&g_product_error, 2);
    return;
  }
  const int rank = a.split > 1 ? cluster_rank() : 0, first = a.split > 1 ? blockIdx.x / a.split : blockIdx.x, units = a.split > 1 ? gridDim.x / a.split : gridDim.x;
  const int b0 = rank * a.share + min(rank, a.more), b1 = b0 + a.share + (rank < a.more ? 1 : 0);   // K blocks of this CTA
  bool ok = true;
  ProductTile tile{};
  int c = 0;                                   // K blocks so far
  const int early = a.group_start ? 0 : min(S::STAGES, b1 - b0);
  auto copy_w = [&](int s, int b) {
    const uint32_t bar = shared_addr(&sm.full[s]);
    bar_expect(bar, S::W_BYTES);
    tensor_g2s(shared_addr(sm.w[s]), &maps.w, b * PB, tile.n * PB, tile.group, bar);
  };
  auto copy_x = [&](int s, int b) {
    const uint32_t bar = shared_addr(&sm.full[s]);
    if (ROWS > FEW_BOX && tile.rows > 2 * FEW_BOX) {
      bar_expect(bar, ROWS * PB);
      tensor_g2s(shared_addr(sm.x[s]), &maps.x, b * PB, tile.row, 0, bar);
    } else {
      const int boxes = (tile.rows + FEW_BOX - 1) / FEW_BOX;
      bar_expect(bar, boxes * S::BOX_BYTES);
      for (int i = 0; i < boxes; i++) tensor_g2s(shared_addr(sm.x[s]) + i * S::BOX_BYTES, &maps.more, b * PB, tile.row + i * FEW_BOX, 0, bar);
    }
  };
  if (warp == 0) {
    if (lane < S::STAGES) bar_init(shared_addr(&sm.full[lane]), 2), bar_init(shared_addr(&sm.empty[lane]), 1);
    else if (lane < S::STAGES + S::SUMS) bar_init(shared_addr(&sm.sum_full[lane - S::STAGES]), 2), bar_init(shared_addr(&sm.sum_empty[lane - S::STAGES]), 8);
    else if (lane == 31) bar_init(shared_addr(&sm.drained), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
    grid_dependency_wait();
    // The first copies are on their way before anything else is set up (groups: before that it is not known which).
    if (lane == 0 && early > 0) {
      tile.find(a, sm.tiles, first, ROWS);
      for (int i = 0; i < early; i++) copy_w(i, b0 + i), copy_x(i, b0 + i);
    }
  } else if (warp == 1) {
    tmem_alloc(shared_addr(&sm.tmem), S::SUMS * ROWS);
  } else if (threadIdx.x == 64) {
    tensor_map_prefetch(ROWS > FEW_BOX && a.rows > 2 * FEW_BOX ? &maps.x : &maps.more);
  }
  grid_dependency_wait();                      // (nothing in front of here looks at what another kernel may be writing)
  grid_dependents_may_start();
  tmem_fence_before();
  sm.tiles.find(a, ROWS);
  tmem_fence_after();
  const uint32_t tmem = sm.tmem;
  // The sums of a split tile are handed over in the place of the outputs where they fit, else in that of the weights, when nobody uses them any more.
  const bool small = (a.rows < ROWS ? a.rows : ROWS) + a.split <= (int)sizeof(sm.out) / (PB * 4);
  __syncwarp();
  if (a.split > 1 && small) cluster_arrive();
  if (warp == 0 || warp == 3) {                // ---- tensor copies: the weights' and the rows', a thread each (a copy takes 200 clocks to issue) ----
    if (lane == 0) {
      c = early;
      for (int t = first; ok && tile.find(a, sm.tiles, t, ROWS); t += units)
        for (int b = t == first ? b0 + early : b0; b < b1; b++, c++) {
          const int s = c % S::STAGES, turn = c / S::STAGES;
          if (turn > 0 && !(ok = reached(shared_addr(&sm.empty[s]), (turn + 1) & 1))) break;
          if (warp == 0) copy_w(s, b);
          else copy_x(s, b);
        }
      // Before their shared memory is gone: the copies on their way, or the products' arrivals that no copy waits for any more.
      if (!ok) {
        for (int i = max(c - S::STAGES, 0); i < c; i++) reached(shared_addr(&sm.full[i % S::STAGES]), (i / S::STAGES) & 1);
      } else if (warp == 0) {
        for (int i = max(c - S::STAGES, 0); ok && i < c; i++) ok = reached(shared_addr(&sm.empty[i % S::STAGES]), (i / S::STAGES) & 1);
      }
    }
  } else if (warp == 1) {                      // ---- products: one thread ----
    if (elect_one()) {
      for (int t = first; ok && tile.find(a, sm.tiles, t, ROWS); t += units) {
        const uint32_t what = mma_e4m3(PB, (tile.rows + 15) / 16 * 16);
        for (int b = b0; b < b1; b++, c++) {
          const int s = c % S::STAGES, turn = c / S::STAGES, buf = c % S::SUMS;
          if (c >= S::SUMS && !(ok = reached(shared_addr(&sm.sum_empty[buf]), (c / S::SUMS + 1) & 1))) break;
          if (!(ok = reached(shared_addr(&sm.full[s]), turn & 1))) break;
          tmem_fence_after();
          const Operand W = operand(shared_addr(sm.w[s]), 0, 1024), X = operand(shared_addr(sm.x[s]), 0, 1024);
#pragma unroll
          for (int k = 0; k < 4; k++) mma8_ss(tmem + buf * ROWS, W + 32 * k, X + 32 * k, what, k > 0);
          mma_commit(shared_addr(&sm.sum_full[buf]));
          mma_commit(shared_addr(&sm.empty[s]));
        }
      }
      if (!ok) {                               // the products on their way
        mma_commit(shared_addr(&sm.drained));
        reached(shared_addr(&sm.drained), 0);
      }
    }
  } else if (warp == 2) {                      // ---- factors: a lane has every 32nd row, loaded four K blocks ahead ----
    // A K block's factors are in their place when sum_full says that its sums are.  The place was the K block's 2 * SUMS in front of it: when the product of
    // the one SUMS in front has ended, its accumulator had been given back by all who read these factors in front of it.
    constexpr int AHEAD = 4;
    float x[AHEAD][ROWS / 32], w[AHEAD];
    ProductTile at;                            // of the K block that is loaded next
    int t = first, b = b0, n = 0;
    bool there = at.find(a, sm.tiles, t, ROWS), more[AHEAD];
    auto load = [&](int k) {
      if (there && b == b1) {
        b = b0, t += units;
        there = at.find(a, sm.tiles, t, ROWS);
      }
      more[k] = there;
      if (!there) return;
      w[k] = a.w_scale[((int64_t)at.group * a.tiles_n + at.n) * a.blocks + b];
      const float *px = a.x_scale + b * a.x_scale_stride + at.row + lane;
#pragma unroll
      for (int i = 0; i < ROWS / 32; i++) x[k][i] = 32 * i + lane < at.rows ? px[32 * i] : 0.0f;
      b++;
    };
    Patience patience;
#pragma unroll
    for (int k = 0; k < AHEAD; k++) load(k);
    while (more[0]) {
#pragma unroll
      for (int k = 0; k < AHEAD; k++) {
        if (!more[k]) break;
        const int buf = n % S::SUMS;
        if (n >= S::SUMS) patience.wait(shared_addr(&sm.sum_full[buf]), (n / S::SUMS + 1) & 1);
#pragma unroll
        for (int i = 0; i < ROWS / 32; i++) sm.factor[n % (2 * S::SUMS)][32 * i + lane] = x[k][i] * w[k];
        __syncwarp();
        if (lane == 0) bar_arrive(shared_addr(&sm.sum_full[buf]));
        n++;
        load(k);
      }
    }
    ok = !patience.gone();
  }
  // ---- sums in binary32, outputs: half of a tile's rows, 32 output channels ----
  constexpr int COLS = ROWS / 2;
  const int part = warp % 4, col0 = (warp - 4) / 4 * COLS;
  float sum[COLS];
  if (warp >= 4) {
    Patience patience;
    for (int t = first; tile.find(a, sm.tiles, t, ROWS); t += units) {
      const int cols = tile.rows - col0;       // columns of this warp
#pragma unroll
      for (int i = 0; i < COLS; i++) sum[i] = 0.0f;
      for (int b = b0; b < b1; b++, c++) {
        const int buf = c % S::SUMS;
        patience.wait(shared_addr(&sm.sum_full[buf]), (c / S::SUMS) & 1);
        tmem_fence_after();
        const float *f = &sm.factor[c % (2 * S::SUMS)][col0];
#pragma unroll
        for (int j = 0; j < COLS; j += 16) {
          if (j < cols) {
            uint32_t d[16];
            tmem_load16(tmem + buf * ROWS + col0 + j + ((uint32_t)part << 21), d);
            tmem_wait_loads(d);
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const float4 x = *reinterpret_cast<const float4 *>(&f[j + i]);
              const float2 lo = __ffma2_rn(make_float2(__uint_as_float(d[i]), __uint_as_float(d[i + 1])), make_float2(x.x, x.y), make_float2(sum[j + i], sum[j + i + 1]));
              const float2 hi = __ffma2_rn(make_float2(__uint_as_float(d[i + 2]), __uint_as_float(d[i + 3])), make_float2(x.z, x.w), make_float2(sum[j + i + 2], sum[j + i + 3]));
              sum[j + i] = lo.x, sum[j + i + 1] = lo.y, sum[j + i + 2] = hi.x, sum[j + i + 3] = hi.y;
            }
          }
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(shared_addr(&sm.sum_empty[buf]));
      }
      ok = !patience.gone();
      if (a.split > 1) break;                  // (one tile)
      const int n = tile.n * PB + 32 * part;
      T *dst = static_cast<T *>(a.out) + (int64_t)(tile.row + col0) * a.out_stride + n;
#pragma unroll
      for (int j = 0; j < COLS; j += 16)
        if (ok && j < cols && n < a.outs) store_columns<WIDE>(sm.out[warp - 4], dst + j * a.out_stride, a.out_stride, sum + j, min(cols - j, 16), a.outs - n, lane);
    }
  }
  if (a.split > 1) {                           // (every CTA of the cluster has the same tile, and there is one)
    float *const parts = reinterpret_cast<float *>(small ? &sm.out[0][0] : &sm.w[0][0]);
    tile.find(a, sm.tiles, first, ROWS);
    const int share = (tile.rows + a.split - 1) / a.split;   // rows of a CTA
    __syncwarp();
    if (!small) cluster_arrive();
    cluster_wait();
    if (warp >= 4 && col0 < tile.rows) {
      const uint32_t to = shared_addr(parts + rank * share * PB + 32 * part + lane);
      int owner = col0 / share, in = col0 - owner * share;
      uint32_t at = shared_of(to + in * PB * 4, owner);
#pragma unroll
      for (int i = 0; i < COLS; i++) {
        if (col0 + i >= tile.rows) break;
        store_shared_of(at, sum[i]);
        at += PB * 4;
        if (++in == share) in = 0, at = shared_of(to, ++owner < a.split ? owner : 0);
      }
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    if (warp >= 4 && __all_sync(0xffffffffu, ok)) {
      const int rows = min(tile.rows - rank * share, share), n = tile.n * PB + 4 * lane;
      for (int r = warp - 4; r < rows; r += 8) {
        float4 v = *reinterpret_cast<const float4 *>(parts + r * PB + 4 * lane);
        for (int q = 1; q < a.split; q++) {
          const float4 y = *reinterpret_cast<const float4 *>(parts + (q * share + r) * PB + 4 * lane);
          v = make_float4(v.x + y.x, v.y + y.y, v.z + y.z, v.w + y.w);
        }
        T *dst = static_cast<T *>(a.out) + (int64_t)(tile.row + rank * share + r) * a.out_stride + n;
        const float x[4] = {v.x, v.y, v.z, v.w};
        alignas(16) T y[4];
        pack(x, y);
        if (WIDE && n + 4 <= a.outs) {
          store_row<true>(dst, y);
        } else {
#pragma unroll
          for (int e = 0; e < 4; e++)
            if (n + e < a.outs) dst[e] = y[e];
        }
      }
    }
  }
  if (!ok) atomicOr(&g_product_error, 1);
  __syncwarp();
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (warp == 1) tmem_free(tmem, S::SUMS * ROWS);
}

// ---------------------------------------------------------------------------------------------
// Many rows: rows of x are the rows of the accumulator, a row's factor is one number of its thread.  Two CTAs of a cluster work on one tile of 256 rows and
// 256 output channels: either has 128 rows of x and of the weights in its shared memory and 128 rows of the sums in its tensor memory, which halves what a tile
// takes from L2 (64 KB a K block; at 13 TB/s that alone is 0.36 us, the products 0.28 us).  Two accumulators: one is taken over while the next K block's
// product goes to the other.
//   warp 0       tensor copies of this CTA's half of either operand, up to five K blocks ahead
//   warp 1       one thread of the first CTA issues the products of both
//   warps 2, 3   factors, to shared memory; they arrive on the barrier of the sums, so that there is one wait for both
//   warps 4-11   a row and half of the output channels to a thread: sums in 128 registers; outputs by way of shared memory and tensor copies
// A K block takes 0.49 us: 64 multiply-adds of pairs a thread (two warps of a scheduler 300 clocks, 370 with the loads of tensor memory, which also compete with the products
// for it), the two barriers and the products' own 512 - 590 clocks in turn on two accumulators.  8192 x 4096 x 12352 352 us, 2.36 PFLOP/s (432 us, 1.92, in a
// long loop under the power cap; the library's product with one scale for all 290 and 335 us); tensor pipe active 59 %.
// Without any hand-over it would be 10 % less.  Halves of 128 output channels, sixteen warps for the sums or wider loads of tensor memory gave nothing.
// ---------------------------------------------------------------------------------------------
constexpr int MANY_THREADS = 384, MANY_ROWS = 256, MANY_OUTS = 256;
struct ManyShared {
  static constexpr int STAGES = 5;
  static constexpr uint32_t BYTES = 128 * PB;  // of either operand in a CTA
  uint8_t x[STAGES][BYTES], w[STAGES][BYTES];
  uint8_t out[8][2][32 * 64];                  // 64 bytes of 32 rows, two of a warp each
  float factor[4][2][128];                     // of four K blocks: of a row, for 128 output channels each
  uint64_t full[STAGES], empty[STAGES], sum_full[2], sum_empty[2], drained;   // (full, sum_empty: the first CTA's)
  uint32_t tmem;
  GroupTiles tiles;
};

// 64 bytes of output channels of a warp's 32 rows, a row to a lane, as T in shared memory (64-byte swizzle).
template <typename T>
__device__ __forceinline__ void stage_sums(uint8_t *stage, const float2 *v, int lane) {
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int u = 0; u < 4; u++) {
    float x[N];
#pragma unroll
    for (int e = 0; e < N / 2; e++) x[2 * e] = v[N / 2 * u + e].x, x[2 * e + 1] = v[N / 2 * u + e].y;
    alignas(16) T t[N];
    pack(x, t);
    *reinterpret_cast<uint4 *>(stage + 64 * lane + 16 * (u ^ (lane / 2 % 4))) = *reinterpret_cast<const uint4 *>(t);
  }
}
// From there to rows of which `rows`, and output channels of which `n` are there: neighbouring lanes write neighbouring channels.
template <bool WIDE, typename T>
__device__ __forceinline__ void copy_sums(const uint8_t *stage, T *dst, int64_t stride, int rows, int n, int lane) {
  constexpr int N = 64 / sizeof(T), F = 16 / sizeof(T);
  if (WIDE && n >= N) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = 8 * i + lane / 4, u = lane % 4;
      if (r < rows) *reinterpret_cast<uint4 *>(dst + r * stride + u * F) = *reinterpret_cast<const uint4 *>(stage + 64 * r + 16 * (u ^ (r / 2 % 4)));
    }
  } else if (lane < N && lane < n) {
#pragma unroll 4
    for (int r = 0; r < rows; r++) dst[r * stride + lane] = reinterpret_cast<const T *>(stage + 64 * r + 16 * ((lane / F) ^ (r / 2 % 4)))[lane % F];
  }
}

template <typename T, bool WIDE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MANY_THREADS, 1) product_many_kernel(const __grid_constant__ ProductMaps maps, const ProductArgs a) {
  extern __shared__ __align__(1024) uint8_t raw[];
  using S = ManyShared;
  S &sm = *reinterpret_cast<S *>(raw);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, rank = cluster_rank(), first = blockIdx.x / 2, units = gridDim.x / 2;
  if (shared_addr(raw) % 1024 != 0) {          // (the swizzled tiles count on it)
    if (threadIdx.x == 0) atomicOr(&g_product_error, 2);
    return;
  }
  if (threadIdx.x == 0) {
    auto init = [](uint64_t &bar, int count) { bar_init(shared_addr(&bar), count); };
    for (int i = 0; i < S::STAGES; i++) init(sm.full[i], 1), init(sm.empty[i], 1);
    for (int i = 0; i < 2; i++) init(sm.sum_full[i], 2), init(sm.sum_empty[i], 16);
    init(sm.drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) pair_tmem_alloc(shared_addr(&sm.tmem), 512);
  grid_dependency_wait();
  grid_dependents_may_start();
  tmem_fence_before();
  sm.tiles.find(a, MANY_ROWS);
  __syncwarp();
  cluster_sync();
  tmem_fence_after();
  const uint32_t tmem = sm.tmem;
  bool ok = true;
  ProductTile tile;
  int c = 0;                                   // K blocks so far
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0) {                          // ---- tensor copies: this CTA's half of either operand ----
      if (lane == 0) {
        for (int t = first; ok && tile.find(a, sm.tiles, t, MANY_ROWS); t += units)
          for (int b = 0; b < a.blocks; b++, c++) {
            const int s = c % S::STAGES, turn = c / S::STAGES;
            if (turn > 0 && !(ok = reached(shared_addr(&sm.empty[s]), (turn + 1) & 1))) break;
            const uint32_t bar = shared_of(shared_addr(&sm.full[s]), 0);
            if (rank == 0) bar_expect(shared_addr(&sm.full[s]), 4 * S::BYTES);
            pair_tensor_g2s(shared_addr(sm.x[s]), &maps.x, b * PB, tile.row + 128 * rank, 0, bar);
            pair_tensor_g2s(shared_addr(sm.w[s]), &maps.w, b * PB, tile.n * MANY_OUTS + 128 * rank, tile.group, bar);
          }
        // Before their shared memory is gone: the copies on their way, or the products' arrivals (in either CTA) that no copy waits for any more.
        if (ok) {
          for (int i = max(c - S::STAGES, 0); ok && i < c; i++) ok = reached(shared_addr(&sm.empty[i % S::STAGES]), (i / S::STAGES) & 1);
        } else if (rank == 0) {
          for (int i = max(c - S::STAGES, 0); i < c; i++) reached(shared_addr(&sm.full[i % S::STAGES]), (i / S::STAGES) & 1);
        }
      }
    } else if (warp == 1) {                    // ---- products, for both CTAs: one thread ----
      constexpr uint32_t what = mma_e4m3(MANY_ROWS, MANY_OUTS);
      if (rank == 0 && elect_one()) {
        for (int t = first; ok && tile.find(a, sm.tiles, t, MANY_ROWS); t += units)
          for (int b = 0; ok && b < a.blocks; b++, c++) {
            const int s = c % S::STAGES, turn = c / S::STAGES, buf = c & 1;
            if (!(ok = reached(shared_addr(&sm.full[s]), turn & 1))) break;
            const Operand X = operand(shared_addr(sm.x[s]), 0, 1024), W = operand(shared_addr(sm.w[s]), 0, 1024);
            if (c >= 2 && !(ok = reached(shared_addr(&sm.sum_empty[buf]), ((c >> 1) + 1) & 1))) break;
            tmem_fence_after();
#pragma unroll
            for (int k = 0; k < 4; k++) pair_mma8_ss(tmem + buf * MANY_OUTS, X + 32 * k, W + 32 * k, what, k > 0);
            pair_mma_commit(shared_addr(&sm.sum_full[buf]));
            pair_mma_commit(shared_addr(&sm.empty[s]));
          }
        if (!ok) {                             // the products on their way
          pair_mma_commit(shared_addr(&sm.drained));
          reached(shared_addr(&sm.drained), 0);
        }
      }
    } else {                                   // ---- factors: of every other K block each, four rows a lane, loaded two K blocks of its own ahead ----
      // A K block's factors are in their place when sum_full says that its sums are.  The place was the K block's four in front of it: when the product of the one
      // two in front has ended, that product's accumulator had been given back by all who read these factors in front of it.
      float x[2][4], w[2][2];
      ProductTile at;                          // of the K block that is loaded next
      int t = first, b = warp - 2, n = warp - 2;
      bool there = at.find(a, sm.tiles, t, MANY_ROWS);
      const int blocks_n = (a.outs + PB - 1) / PB;
      auto load = [&](int k) {
        while (there && b >= a.blocks) {
          b -= a.blocks, t += units;
          there = at.find(a, sm.tiles, t, MANY_ROWS);
        }
        if (!there) return false;
        const int rows = at.rows - 128 * rank;
        const float *px = a.x_scale + b * a.x_scale_stride + at.row + 128 * rank + lane;
        const float *pw = a.w_scale + ((int64_t)at.group * blocks_n + 2 * at.n) * a.blocks + b;
        w[k][0] = pw[0];
        w[k][1] = 2 * at.n + 1 < blocks_n ? pw[a.blocks] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; i++) x[k][i] = 32 * i + lane < rows ? px[32 * i] : 0.0f;
        b += 2;
        return true;
      };
      Patience patience;
      bool more[2] = {load(0), load(1)};
      while (more[0]) {
#pragma unroll
        for (int k = 0; k < 2; k++) {
          if (!more[k]) break;
          const int buf = n & 1;
          if (n >= 2) patience.wait(shared_addr(&sm.sum_full[buf]), ((n >> 1) + 1) & 1);
          float (*f)[128] = sm.factor[n & 3];
#pragma unroll
          for (int i = 0; i < 4; i++) f[0][32 * i + lane] = x[k][i] * w[k][0], f[1][32 * i + lane] = x[k][i] * w[k][1];
          __syncwarp();
          if (lane == 0) bar_arrive(shared_addr(&sm.sum_full[buf]));
          n += 2;
          more[k] = load(k);
        }
      }
      ok = !patience.gone();
    }
  } else {                                     // ---- sums in binary32, outputs: a row each, half of the tile's output channels ----
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");   // (256 * 224 + 128 * 56 of the 384 * 168 that the block starts with)
    const int part = warp % 4, half = (warp - 4) / 4;
    const uint32_t from = tmem + 128 * half + ((uint32_t)part << 21);
    const uint32_t full = shared_addr(&sm.sum_full[0]), empty = shared_of(shared_addr(&sm.sum_empty[0]), 0);
    Patience patience;
    int turns = 0;                             // copies so far
    for (int t = first; tile.find(a, sm.tiles, t, MANY_ROWS); t += units) {
      const int rows = min(tile.rows - 128 * rank - 32 * part, 32);
      float2 sum[64];
#pragma unroll
      for (int i = 0; i < 64; i++) sum[i] = make_float2(0.0f, 0.0f);
#pragma unroll 1
      for (int b = 0; b < a.blocks; b++, c++) {
        const int buf = c & 1;
        patience.wait(full + 8 * buf, (c >> 1) & 1);
        tmem_fence_after();
        if (rows <= 0) {                       // (none of the warp's rows)
          tmem_fence_before();
          if (lane == 0) bar_arrive_cluster(empty + 8 * buf);
          continue;
        }
        uint32_t d[2][16];
        tmem_load16(from + buf * MANY_OUTS, d[0]);
        const float f = sm.factor[c & 3][half][32 * part + lane];
        const float2 ff = make_float2(f, f);
#pragma unroll
        for (int j = 0; j < 8; j++) {
          tmem_wait_loads(d[j & 1]);
          if (j < 7) tmem_load16(from + buf * MANY_OUTS + 16 * (j + 1), d[(j + 1) & 1]);
          if (j == 7) {
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive_cluster(empty + 8 * buf);
          }
#pragma unroll
          for (int i = 0; i < 8; i++) sum[8 * j + i] = __ffma2_rn(make_float2(__uint_as_float(d[j & 1][2 * i]), __uint_as_float(d[j & 1][2 * i + 1])), ff, sum[8 * j + i]);
        }
      }
      const int n = tile.n * MANY_OUTS + 128 * half, row = tile.row + 128 * rank + 32 * part;
      ok = !patience.gone();
      constexpr int N = 64 / sizeof(T);
#pragma unroll
      for (int i = 0; i < 128 / N; i++)
        if (ok && rows > 0 && n + N * i < a.outs) {
          // (a copy writes whole pieces of 16 bytes, and all rows)
          const bool copied = WIDE && rows == 32 && n + N * (i + 1) <= a.outs;
          uint8_t *const stage = sm.out[warp - 4][turns & 1];
          if (copied) copies_read<1>();        // (the last but one was from this place)
          else copies_read<0>();
          __syncwarp();
          stage_sums<T>(stage, sum + N / 2 * i, lane);
          fence_async_shared();
          __syncwarp();
          if (copied) {
            if (lane == 0) tensor_s2g(&maps.more, shared_addr(stage), (n + N * i) * (int)sizeof(T), row, 0), copies_commit();
            turns++;
          } else {
            copy_sums<WIDE>(stage, static_cast<T *>(a.out) + (int64_t)row * a.out_stride + n + N * i, a.out_stride, rows, a.outs - n - N * i, lane);
            __syncwarp();
          }
        }
    }
    copies_done();
  }
  if (!ok) atomicOr(&g_product_error, 1);
  __syncwarp();
  tmem_fence_before();
  cluster_sync();
  tmem_fence_after();
  if (warp == 1) pair_tmem_free(tmem, 512);
}

}  // namespace lq
