// C boundary of the operators around the decode step: argument checks and launches.  Declarations and contracts: include/lq.h.
#include <algorithm>
#include <atomic>
#include <initializer_list>

#include "lq_conv.cuh"
#include "lq_norm.cuh"
#include "lq_scan.cuh"

namespace lq {

static cudaStream_t cuda_stream(lq_stream s) { return reinterpret_cast<cudaStream_t>(s); }

static bool aligned(const void *p, unsigned bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

static lq_status launched() { return cudaGetLastError() == cudaSuccess ? LQ_OK : LQ_ERR_CUDA; }

static unsigned type_size(int type) { return type == LQ_F32 ? 4 : 2; }

static long ceil_div(long a, long b) { return (a + b - 1) / b; }

static bool bad_count(int n) { return n < 0; }

// Row and sequence numbers up to a tile or a CTA beyond the last one are formed in 32 bits.
constexpr int MOST_ROWS = INT32_MAX - 1023;

// Required and optional (may be null) arrays with elements of `bytes` bytes.
static lq_status check_arrays(unsigned bytes, std::initializer_list<const void *> required, std::initializer_list<const void *> optional = {}) {
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
static bool rows_overlap(const void *a, int64_t sa, long wa, const void *b, int64_t sb, long wb, long rows, unsigned bytes) {
  if (rows <= 0) return false;
  const intptr_t x = reinterpret_cast<intptr_t>(a), y = reinterpret_cast<intptr_t>(b);
  const intptr_t ex = x + ((rows - 1) * sa + wa) * (intptr_t)bytes, ey = y + ((rows - 1) * sb + wb) * (intptr_t)bytes;
  if (ex <= y || ey <= x) return false;
  if (sa != sb) return true;
  const intptr_t period = sa * (intptr_t)bytes, d = ((y - x) % period + period) % period;   // b's rows start d bytes into a's
  return d < wa * (intptr_t)bytes || d + wb * (intptr_t)bytes > period;
}

// Whether `bytes` bytes at p, without gaps, meet the range of those strided rows.
static bool meets_rows(const void *p, uint64_t bytes, const void *a, int64_t sa, long wa, long rows, unsigned size) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(a);
  return rows > 0 && x < y + ((rows - 1) * (uint64_t)sa + wa) * size && y < x + bytes;
}

// ---- short causal convolution ----

static lq_status check_conv(const lq_conv *s, bool step) {
  if (!s) return LQ_ERR_NULL;
  if (bad_count(s->tokens) || bad_count(s->seqs) || s->channels <= 0 || s->width <= 0 || bad_count(s->n_slots)) return LQ_ERR_SHAPE;
  if (s->type < LQ_BF16 || s->type > LQ_F32 || (s->silu != 0 && s->silu != 1)) return LQ_ERR_SHAPE;
  if (step && s->tokens != s->seqs) return LQ_ERR_SHAPE;
  if (s->width < 2 || s->width > 4 || s->tokens > MOST_ROWS || s->seqs > MOST_ROWS) return LQ_ERR_UNSUPPORTED;
  return LQ_OK;
}

template <typename T, int W, int VEC>
static lq_status launch_conv_t(const lq_conv *s, ConvArgs a, bool step, cudaStream_t stream) {
  const long blocks_c = ceil_div(s->channels, CONV_THREADS * VEC);
  a.blocks_c = (int)blocks_c;
  if (step) {
    if (blocks_c * s->seqs > INT32_MAX) return LQ_ERR_UNSUPPORTED;
    conv_step_kernel<T, W, VEC><<<blocks_c * s->seqs, CONV_THREADS, 0, stream>>>(a);
  } else {
    // The largest tile that leaves three CTAs to an SM; 128 rows only for 16-bit types and twelve CTAs to an SM.  8192 channels, bf16: 32768
    // rows in tiles of 128, 64, 32, 16, 8 take 192, 200, 217, 285, 426 us; 16384 rows 102, 106, 115, 147; 8192 rows 63, 59, 65, 80; 1024 rows in
    // 64, 32, 16, 8 16.4, 16.4, 16.4, 18.4; 128 rows 12.3, 10.2, 8.2, 8.2; binary32, 16384 rows in 128, 64, 32: 190, 182, 190.
    a.rows_per_tile = sizeof(T) == 2 && ceil_div(s->tokens, 128) * blocks_c >= 12 * 148 ? 128 : 64;
    while (a.rows_per_tile > 8 && ceil_div(s->tokens, a.rows_per_tile) * blocks_c < 3 * 148) a.rows_per_tile /= 2;
    const long grid = ceil_div(s->tokens, a.rows_per_tile) * blocks_c;
    if (grid > INT32_MAX) return LQ_ERR_UNSUPPORTED;
    conv_prompt_kernel<T, W, VEC><<<grid, CONV_THREADS, 0, stream>>>(a);
  }
  return launched();
}

template <typename T>
static lq_status launch_conv(const lq_conv *s, const ConvArgs &a, bool step, cudaStream_t stream) {
  constexpr int VEC = 4;
  bool wide = s->channels % VEC == 0 && a.x_stride % VEC == 0 && a.out_stride % VEC == 0 && aligned(a.w, 16);
  for (const void *p : {a.x, (const void *)a.state, (const void *)a.out}) wide = wide && aligned(p, VEC * sizeof(T));
#define LQ_CONV(W) return wide ? launch_conv_t<T, W, VEC>(s, a, step, stream) : launch_conv_t<T, W, 1>(s, a, step, stream)
  if (s->width == 2) LQ_CONV(2);
  if (s->width == 3) LQ_CONV(3);
  LQ_CONV(4);
#undef LQ_CONV
}

static lq_status conv(const lq_conv *s, const void *x, int64_t x_stride, const void *w, const void *bias, void *state, void *out,
                      int64_t out_stride, const int32_t *seq_start, const int32_t *slots, const int32_t *resume, bool step,
                      lq_stream stream) {
  lq_status rc = check_conv(s, step);
  if (rc != LQ_OK) return rc;
  if (s->tokens == 0 || s->seqs == 0) return LQ_OK;
  const unsigned bytes = type_size(s->type);
  if ((rc = check_arrays(bytes, {x, w, out}, {bias, state})) != LQ_OK) return rc;
  if ((rc = check_arrays(4, {}, {seq_start, slots, resume})) != LQ_OK) return rc;
  if (step ? !state : !seq_start) return LQ_ERR_NULL;
  if (!step && resume && !state) return LQ_ERR_NULL;
  if (x_stride < s->channels || out_stride < s->channels) return LQ_ERR_SHAPE;
  if (!(step && x == out && x_stride == out_stride) &&
      rows_overlap(x, x_stride, s->channels, out, out_stride, s->channels, s->tokens, bytes))
    return LQ_ERR_UNSUPPORTED;
  const uint64_t states = state ? (uint64_t)s->n_slots * (s->width - 1) * s->channels * bytes : 0;
  if (meets_rows(state, states, x, x_stride, s->channels, s->tokens, bytes) || meets_rows(state, states, out, out_stride, s->channels, s->tokens, bytes))
    return LQ_ERR_UNSUPPORTED;
  ConvArgs a{x, w, bias, state, out, x_stride, out_stride, {seq_start, slots, resume, s->tokens, s->seqs, state ? s->n_slots : INT32_MAX},
             s->channels, s->silu, 0, 0};
  if (s->type == LQ_F32) return launch_conv<float>(s, a, step, cuda_stream(stream));
  if (s->type == LQ_F16) return launch_conv<__half>(s, a, step, cuda_stream(stream));
  return launch_conv<__nv_bfloat16>(s, a, step, cuda_stream(stream));
}

// ---- norms of queries and keys with the rotation ----

template <typename T, int DIM>
static lq_status launch_norm_t(const lq_norm *s, NormArgs a, bool wide, cudaStream_t stream) {
  // as many rows to a CTA as keep its lanes busy for some trips, and not more than leave two CTAs to an SM
  const long heads = s->heads_q + s->heads_k, lanes = NORM_THREADS / (DIM * (long)sizeof(T) / 32);
  a.rows_per_cta = (int)std::max(1l, std::min({(long)NORM_MAX_ROWS, std::max(1l, NORM_TRIPS * lanes / heads), s->tokens / (2 * 148l)}));
  const long grid = ceil_div(s->tokens, a.rows_per_cta);
  if (wide) norm_rotate_kernel<T, DIM, true><<<grid, NORM_THREADS, 0, stream>>>(a);
  else norm_rotate_kernel<T, DIM, false><<<grid, NORM_THREADS, 0, stream>>>(a);
  return launched();
}

template <typename T>
static lq_status launch_norm(const lq_norm *s, const NormArgs &a, cudaStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  bool wide = true;
  for (const void *p : {a.q, a.k, (const void *)a.out_q, (const void *)a.out_k}) wide = wide && aligned(p, 16);
  for (int64_t stride : {a.q_stride, a.k_stride, a.out_q_stride, a.out_k_stride}) wide = wide && stride % VEC == 0;
  if (s->dim == 64) return launch_norm_t<T, 64>(s, a, wide, stream);
  if (s->dim == 128) return launch_norm_t<T, 128>(s, a, wide, stream);
  return launch_norm_t<T, 256>(s, a, wide, stream);
}

// ---- selective scan ----

static lq_status check_scan(const lq_scan *s, bool step) {
  if (!s) return LQ_ERR_NULL;
  if (bad_count(s->tokens) || bad_count(s->seqs) || bad_count(s->n_slots) || s->heads_v <= 0 || s->heads_qk <= 0 || s->d_k <= 0 || s->d_v <= 0)
    return LQ_ERR_SHAPE;
  if (s->heads_v % s->heads_qk != 0 || (s->select != 0 && s->select != 1)) return LQ_ERR_SHAPE;
  if (step ? s->tokens != s->seqs : s->max_len < 0) return LQ_ERR_SHAPE;
  if (s->gate_type != LQ_BF16 && s->gate_type != LQ_F32) return LQ_ERR_UNSUPPORTED;
  // (2^30 heads: numbers of items go on beyond the last one by as many as there are CTAs)
  if (s->d_k != SD || s->d_v != SD || s->tokens > MOST_ROWS || (long)s->seqs * s->heads_v > 1 << 30) return LQ_ERR_UNSUPPORTED;
  return LQ_OK;
}

static lq_status check_scan_io(const lq_scan *s, const lq_scan_io *io, const void *o, int64_t o_stride, bool step) {
  lq_status rc;
  if (!io) return LQ_ERR_NULL;
  if ((rc = check_arrays(16, {io->S}, {io->S0})) != LQ_OK) return rc;
  if (!step && !io->seq_start) return LQ_ERR_NULL;
  if ((rc = check_arrays(4, {}, {io->A, io->dt_bias, io->skip, io->seq_start, io->slots, io->resume})) != LQ_OK) return rc;
  const uint64_t states = (uint64_t)s->n_slots * s->heads_v * (SD * SD) * sizeof(float);
  if (io->S0 && io->S0 != io->S && meets_rows(io->S, states, io->S0, 0, (long)states, 1, 1)) return LQ_ERR_UNSUPPORTED;
  if (s->tokens == 0) return LQ_OK;
  if ((rc = check_arrays(16, {io->q, io->k, io->v, o})) != LQ_OK) return rc;
  if ((rc = check_arrays(type_size(s->gate_type), {io->beta}, {io->alpha})) != LQ_OK) return rc;
  if (s->select ? !io->A : !io->alpha) return LQ_ERR_NULL;
  const int64_t wq = (int64_t)s->heads_qk * SD, wv = (int64_t)s->heads_v * SD;
  if (io->q_stride < wq || io->k_stride < wq || io->v_stride < wv || o_stride < wv) return LQ_ERR_SHAPE;
  if (io->beta_stride < s->heads_v || (!s->select && io->alpha_stride < s->heads_v)) return LQ_ERR_SHAPE;
  if (io->q_stride % 8 || io->k_stride % 8 || io->v_stride % 8 || o_stride % 8) return LQ_ERR_ALIGN;
  // (the heads of a group, and the blocks' other roles, read q, k and v after the first outputs are written)
  const unsigned size = step ? sizeof(float) : 2;   // of an output
  if (rows_overlap(io->q, io->q_stride * 2, wq * 2, o, o_stride * size, wv * size, s->tokens, 1) ||
      rows_overlap(io->k, io->k_stride * 2, wq * 2, o, o_stride * size, wv * size, s->tokens, 1) ||
      rows_overlap(io->v, io->v_stride * 2, wv * 2, o, o_stride * size, wv * size, s->tokens, 1))
    return LQ_ERR_UNSUPPORTED;
  if (meets_rows(io->S, states, o, o_stride, wv, s->tokens, size) || meets_rows(io->S, states, io->q, io->q_stride, wq, s->tokens, 2) ||
      meets_rows(io->S, states, io->k, io->k_stride, wq, s->tokens, 2) || meets_rows(io->S, states, io->v, io->v_stride, wv, s->tokens, 2))
    return LQ_ERR_UNSUPPORTED;
  if (io->S0 && meets_rows(io->S0, states, o, o_stride, wv, s->tokens, size)) return LQ_ERR_UNSUPPORTED;
  return LQ_OK;
}

static ScanArgs scan_args(const lq_scan *s, const lq_scan_io *io, void *o, int64_t o_stride) {
  auto bf = [](const uint16_t *p) { return reinterpret_cast<const __nv_bfloat16 *>(p); };
  return {bf(io->q), bf(io->k), bf(io->v), io->q_stride, io->k_stride, io->v_stride, io->beta_stride, io->alpha_stride, o_stride, io->beta, io->alpha,
          io->A, io->dt_bias, io->skip, io->S0 ? io->S0 : io->S, io->S, o, {io->seq_start, io->slots, io->resume, s->tokens, s->seqs, s->n_slots}, s->heads_v,
          s->heads_qk, s->max_len < s->tokens ? s->max_len : s->tokens, s->select, s->gate_type == LQ_F32};
}

// How a call's prompts are cut.  Uncut, a CTA has all blocks of a head, and few heads keep few SMs busy; in pieces the blocks are gone through
// twice, the first time (all pieces but the last) for the state alone, which takes 0.65 of the time, and a piece costs one and a half blocks
// more.  1 x 16384 rows of 32 heads in 1, 2, 3, 4, 5, 9, 13 pieces: 399, 324, 229, 184, 240, 188, 192 us; 4 x 4096 rows of 32 heads in 1, 2,
// 4 pieces: 117, 195, 198 us.
constexpr int SMS = 148, MOST_ORDERED = 4096;   // (what scan_order_kernel has room for)

static ScanPlan scan_plan(const lq_scan *s, void *work) {
  const long max_len = s->max_len < s->tokens ? s->max_len : s->tokens;
  const long heads = (long)s->seqs * s->heads_v, blocks = max_len > 0 ? ceil_div(max_len, SB) : 1;
  long best = blocks;                          // blocks of a piece
  double least = (double)ceil_div(heads, SMS) * (blocks + 1.5);
  for (long p = 2; p <= 64 && 2 * p <= blocks; p++) {
    const long piece = ceil_div(blocks, p), pieces = ceil_div(blocks, piece);
    const double t = (piece + 1.5) * (ceil_div(heads * pieces, SMS) + 0.65 * ceil_div(heads * (pieces - 1), SMS)) + 3.0;
    if (t < least) least = t, best = piece;
  }
  ScanPlan plan{};
  plan.piece = (int)best * SB;
  plan.pieces = (int)ceil_div(blocks, best);
  plan.items = (int)(heads * plan.pieces);
  plan.heads.set(s->heads_v);
  plan.cuts.set(plan.pieces);
  plan.group.set(s->heads_v / s->heads_qk);
  // More heads than CTAs: whoever is through takes the next, those of long prompts first where one of them can be more than a quarter of a
  // CTA's share (12 prompts, the longest with a quarter of 24000 rows: 258 -> 240 us; 64 prompts of up to 216 rows: 103 -> 109, the
  // additional launch).
  int *at = static_cast<int *>(work);
  if (plan.items > SMS) {
    plan.next = at;
    at += 4;
    const long share = (s->tokens / SB * s->heads_v + heads) / SMS;
    if (s->seqs <= MOST_ORDERED && s->seqs > 1 && 4 * best > share) plan.order = at, at += ceil_div(s->seqs, 4) * 4;
  }
  plan.states = reinterpret_cast<float *>(at);
  plan.decays = plan.states + (size_t)plan.items * (SD * SD);
  return plan;
}

static uint64_t scan_bytes(const lq_scan *s) {
  char base[16];                               // (an address to measure from)
  const ScanPlan plan = scan_plan(s, base);
  const uint64_t front = reinterpret_cast<char *>(plan.states) - base;
  return front + (plan.pieces > 1 ? (uint64_t)plan.items * (SD * SD + 1) * sizeof(float) : 0);
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
    cudaGetLastError();
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

// [rows][heads][128] bf16 with strided rows, copied in boxes of SB rows of 64 channels of one head
static bool row_map(CUtensorMap *map, const void *base, long rows, int heads, int64_t stride) {
  const cuuint64_t size[3] = {SD, (cuuint64_t)heads, (cuuint64_t)rows}, strides[2] = {SD * 2, (cuuint64_t)stride * 2};
  const cuuint32_t box[3] = {SD / 2, 1, SB}, one[3] = {1, 1, 1};
  const EncodeTiled f = encode_tiled();
  return f && f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), size, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool OUT, typename G, bool SELECT>
static lq_status launch_scan_t(const ScanMaps &maps, const ScanArgs &a, const ScanPlan &plan, cudaStream_t stream) {
  constexpr size_t smem = sizeof(ScanShared);
  static std::atomic<uint64_t> ready{0};        // devices on which the kernel has been given its shared memory
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return LQ_ERR_CUDA;
  const uint64_t bit = uint64_t(1) << (device & 63);
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    if (cudaFuncSetAttribute(scan_blocks_kernel<OUT, G, SELECT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
      cudaGetLastError();
      return LQ_ERR_CUDA;
    }
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  if (plan.order) {
    scan_order_kernel<<<1, 1024, 0, stream>>>(a, plan);
    const lq_status rc = launched();
    if (rc != LQ_OK) return rc;
  } else if (plan.next && cudaMemsetAsync(plan.next, 0, sizeof(int), stream) != cudaSuccess) {
    cudaGetLastError();
    return LQ_ERR_CUDA;
  }
  scan_blocks_kernel<OUT, G, SELECT><<<plan.items < SMS ? plan.items : SMS, SCAN_THREADS, smem, stream>>>(maps, a, plan);
  return launched();
}

template <bool OUT>
static lq_status launch_scan(const ScanMaps &maps, const ScanArgs &a, const ScanPlan &plan, cudaStream_t stream) {
  if (a.select) {
    return a.gates_f32 ? launch_scan_t<OUT, float, true>(maps, a, plan, stream) : launch_scan_t<OUT, __nv_bfloat16, true>(maps, a, plan, stream);
  }
  return a.gates_f32 ? launch_scan_t<OUT, float, false>(maps, a, plan, stream) : launch_scan_t<OUT, __nv_bfloat16, false>(maps, a, plan, stream);
}

}  // namespace lq

using namespace lq;

// lq_check_device / lq_clear_device_flags: the flag of the kernels in this file (each source file has device variables of its own)
namespace lq {
bool ops_flags(int *flags) { return cudaMemcpyFromSymbol(flags, g_ops_error, sizeof(int)) == cudaSuccess; }
bool clear_ops_flags() {
  const int zero = 0;
  return cudaMemcpyToSymbol(g_ops_error, &zero, sizeof(int)) == cudaSuccess;
}
}  // namespace lq

extern "C" {

lq_status lq_conv_prompt(const lq_conv *shape, const void *x, int64_t x_stride, const void *w, const void *bias, void *state,
                         void *out, int64_t out_stride, const int32_t *seq_start, const int32_t *slots,
                         const int32_t *resume, lq_stream stream) {
  return conv(shape, x, x_stride, w, bias, state, out, out_stride, seq_start, slots, resume, false, stream);
}

lq_status lq_conv_step(const lq_conv *shape, const void *x, int64_t x_stride, const void *w, const void *bias, void *state,
                       void *out, int64_t out_stride, const int32_t *slots, lq_stream stream) {
  return conv(shape, x, x_stride, w, bias, state, out, out_stride, nullptr, slots, nullptr, true, stream);
}

lq_status lq_norm_rotate(const lq_norm *s, const void *q, int64_t q_stride, const void *k, int64_t k_stride, void *out_q,
                         int64_t out_q_stride, void *out_k, int64_t out_k_stride, const float *w_q, const float *w_k,
                         const int32_t *positions, const float *inv_freq, lq_stream stream) {
  if (!s) return LQ_ERR_NULL;
  if (bad_count(s->tokens) || bad_count(s->heads_q) || bad_count(s->heads_k) || s->dim <= 0 || s->rot < 0 || s->rot > s->dim) return LQ_ERR_SHAPE;
  if (s->norm < LQ_NORM_NONE || s->norm > LQ_NORM_RMS || (s->pairs != 0 && s->pairs != 1) || s->type < LQ_BF16 || s->type > LQ_F32) return LQ_ERR_SHAPE;
  if ((s->dim != 64 && s->dim != 128 && s->dim != 256) || s->rot % 16 != 0) return LQ_ERR_UNSUPPORTED;
  if ((long)s->heads_q + s->heads_k > (1 << 16)) return LQ_ERR_UNSUPPORTED;
  if (s->tokens == 0 || s->heads_q + s->heads_k == 0) return LQ_OK;
  const unsigned bytes = type_size(s->type);
  lq_status rc;
  struct { const void *in; int64_t in_stride; void *out; int64_t out_stride; int heads; } side[2] = {
      {q, q_stride, out_q, out_q_stride, s->heads_q}, {k, k_stride, out_k, out_k_stride, s->heads_k}};
  for (auto &x : side) {
    if (x.heads == 0) {
      x = {nullptr, 0, nullptr, 0, 0};
      continue;
    }
    if ((rc = check_arrays(bytes, {x.in, x.out})) != LQ_OK) return rc;
    if (x.in_stride < (int64_t)x.heads * s->dim || x.out_stride < (int64_t)x.heads * s->dim) return LQ_ERR_SHAPE;
  }
  if ((rc = check_arrays(4, {}, {w_q, w_k, positions, inv_freq})) != LQ_OK) return rc;
  if (s->rot > 0 && (!positions || !inv_freq)) return LQ_ERR_NULL;
  for (auto &out : side)                       // an output may be its own input, and nothing else
    for (auto &in : side) {
      if (!in.heads || !out.heads || (&in == &out && in.in == in.out && in.in_stride == in.out_stride)) continue;
      if (rows_overlap(in.in, in.in_stride, (long)in.heads * s->dim, out.out, out.out_stride, (long)out.heads * s->dim, s->tokens, bytes))
        return LQ_ERR_UNSUPPORTED;
    }
  if (s->heads_q && s->heads_k &&
      rows_overlap(out_q, out_q_stride, (long)s->heads_q * s->dim, out_k, out_k_stride, (long)s->heads_k * s->dim, s->tokens, bytes))
    return LQ_ERR_UNSUPPORTED;
  NormArgs a{side[0].in, side[1].in, side[0].out, side[1].out, side[0].in_stride, side[1].in_stride, side[0].out_stride, side[1].out_stride,
                   w_q, w_k, inv_freq, positions, s->tokens, s->heads_q, s->heads_k, s->rot, s->pairs, s->norm, 0, s->eps, s->scale_q, s->scale_k, {}, {}};
  a.heads.set(s->heads_q + s->heads_k);
  a.half.set(s->rot > 0 ? s->rot / 2 : 1);
  if (s->type == LQ_F32) return launch_norm<float>(s, a, cuda_stream(stream));
  if (s->type == LQ_F16) return launch_norm<__half>(s, a, cuda_stream(stream));
  return launch_norm<__nv_bfloat16>(s, a, cuda_stream(stream));
}

uint64_t lq_scan_prompt_bytes(const lq_scan *s) { return check_scan(s, false) == LQ_OK ? scan_bytes(s) : 0; }

lq_status lq_scan_prompt(const lq_scan *s, const lq_scan_io *io, uint16_t *o, int64_t o_stride, void *work, lq_stream stream) {
  lq_status rc = check_scan(s, false);
  if (rc != LQ_OK) return rc;
  if (s->seqs == 0) return LQ_OK;
  if ((rc = check_scan_io(s, io, o, o_stride, false)) != LQ_OK) return rc;
  const ScanPlan plan = scan_plan(s, work);
  if (scan_bytes(s) > 0 && (rc = check_arrays(16, {work})) != LQ_OK) return rc;
  ScanMaps maps{};
  if (s->tokens > 0 && !(row_map(&maps.q, io->q, s->tokens, s->heads_qk, io->q_stride) && row_map(&maps.k, io->k, s->tokens, s->heads_qk, io->k_stride) &&
                         row_map(&maps.v, io->v, s->tokens, s->heads_v, io->v_stride)))
    return LQ_ERR_CUDA;
  const ScanArgs a = scan_args(s, io, o, o_stride);
  if (plan.pieces > 1) {
    if ((rc = launch_scan<false>(maps, a, plan, cuda_stream(stream))) != LQ_OK) return rc;
    scan_join_kernel<<<s->seqs * s->heads_v * 16, 256, 0, cuda_stream(stream)>>>(a, plan);
    if ((rc = launched()) != LQ_OK) return rc;
  }
  return launch_scan<true>(maps, a, plan, cuda_stream(stream));
}

lq_status lq_scan_step(const lq_scan *s, const lq_scan_io *io, float *o, int64_t o_stride, lq_stream stream) {
  lq_status rc = check_scan(s, true);
  if (rc != LQ_OK) return rc;
  if (s->seqs == 0) return LQ_OK;
  if ((rc = check_scan_io(s, io, o, o_stride, true)) != LQ_OK) return rc;
  scan_step_kernel<<<s->seqs * s->heads_v, 256, 0, cuda_stream(stream)>>>(scan_args(s, io, o, o_stride));
  return launched();
}

}  // extern "C"
