// C boundary of the 8-bit linear layer around the decode step: argument checks and launches.  Declarations and contracts: include/lq.h.
#include <algorithm>
#include <atomic>

#include "lq_host.h"
#include "lq_product.cuh"
#include "lq_rownorm.cuh"

namespace lq {

constexpr int SMS = 148;

// A launch that may begin while the kernel in front of it on the stream is still draining; its kernel executes griddepcontrol.wait before its first access to
// global memory.  cluster: CTAs of a cluster, 0: what the kernel says.
template <typename K, typename... Args>
static lq_status launch_dependent(K kernel, dim3 grid, dim3 block, size_t smem, cudaStream_t stream, int cluster, const Args &...args) {
  cudaLaunchAttribute attrs[2] = {};
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = cluster, attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t config = {};
  config.gridDim = grid, config.blockDim = block, config.dynamicSmemBytes = smem, config.stream = stream;
  config.attrs = attrs, config.numAttrs = cluster > 0 ? 2 : 1;
  if (cudaLaunchKernelEx(&config, kernel, args...) != cudaSuccess) {
    cudaGetLastError();
    return LQ_ERR_CUDA;
  }
  return LQ_OK;
}

// ---- norms ----

// The memory from the first to the last element of an array of strided rows.
struct Span {
  const void *p;
  int64_t stride;
  long width, rows;
  unsigned size;                               // bytes of an element
};
static bool spans_meet(const Span &a, const Span &b) {
  if (!a.p || !b.p) return false;
  if (a.rows == b.rows) return rows_overlap(a.p, a.stride * a.size, a.width * a.size, b.p, b.stride * b.size, b.width * b.size, a.rows, 1);
  return meets_rows(a.p, ((a.rows - 1) * (uint64_t)a.stride + a.width) * a.size, b.p, b.stride, b.width, b.rows, b.size);
}

struct NormIo {
  const void *in[2];                           // x and the residual, or o and z
  int64_t in_stride[2];
  unsigned in_size[2];
  bool written;                                // the second input is an output too
  const float *w;
  long weights;                                // elements of w that are read
  NormOut o;
};

static NormOut norm_out(const lq_norm_io *n) { return {n->out, n->out8, n->scale, n->out_stride, n->out8_stride, n->scale_stride}; }

static lq_status check_norm_io(const NormIo &io, long tokens, long width, int type, bool in_place) {
  lq_status rc;
  const unsigned size = type_size(type);
  if ((rc = check_arrays(io.in_size[0], {io.in[0]})) != LQ_OK) return rc;
  if ((rc = check_arrays(io.in_size[1], {}, {io.in[1]})) != LQ_OK) return rc;
  if ((rc = check_arrays(size, {}, {io.o.out})) != LQ_OK) return rc;
  if ((rc = check_arrays(4, {}, {io.w, io.o.scale})) != LQ_OK) return rc;
  if ((!io.o.out && !io.o.out8) || (io.o.out8 && !io.o.scale)) return LQ_ERR_NULL;
  for (int i = 0; i < 2; i++)
    if (io.in[i] && io.in_stride[i] < width) return LQ_ERR_SHAPE;
  if ((io.o.out && io.o.out_stride < width) || (io.o.out8 && (io.o.out8_stride < width || io.o.scale_stride < tokens))) return LQ_ERR_SHAPE;
  const Span in[2] = {{io.in[0], io.in_stride[0], width, tokens, io.in_size[0]}, {io.in[1], io.in_stride[1], width, tokens, io.in_size[1]}};
  const Span out[3] = {{io.o.out, io.o.out_stride, width, tokens, size},
                       {io.o.out8, io.o.out8_stride, width, tokens, 1},
                       {io.o.out8 ? io.o.scale : nullptr, io.o.scale_stride, tokens, ceil_div(width, 128), 4}};
  const Span w{io.weights ? io.w : nullptr, io.weights, io.weights, 1, 4};
  if (io.written && (spans_meet(in[0], in[1]) || spans_meet(w, in[1]))) return LQ_ERR_UNSUPPORTED;
  for (int i = 0; i < 3; i++) {
    for (int j = 0; j < 2; j++)
      if (!(in_place && i == 0 && j == 0 && out[0].p == in[0].p && out[0].stride == in[0].stride) && spans_meet(out[i], in[j])) return LQ_ERR_UNSUPPORTED;
    for (int j = 0; j < i; j++)
      if (spans_meet(out[i], out[j])) return LQ_ERR_UNSUPPORTED;
    if (spans_meet(w, out[i])) return LQ_ERR_UNSUPPORTED;
  }
  return LQ_OK;
}

// Whether all rows can be taken in pieces of `line` elements, in steps of 16 bytes.
static bool wide_norm(const NormIo &io, long width, int type, int line) {
  bool wide = width % line == 0 && aligned(io.w, 16) && aligned(io.o.out, 16) && aligned(io.o.out8, line);
  const long elements = 16 / type_size(type);
  for (int i = 0; i < 2; i++) wide = wide && aligned(io.in[i], 16) && (!io.in[i] || io.in_stride[i] % (16 / io.in_size[i]) == 0);
  return wide && (!io.o.out || io.o.out_stride % elements == 0) && (!io.o.out8 || io.o.out8_stride % line == 0);
}

template <typename T, bool WIDE>
static lq_status launch_add(const AddArgs &a, cudaStream_t stream) {
  // two pieces to a thread, one where there are fewer rows than SMs (4096 channels, one row with one, two, four pieces: 2.2, 2.5, 3.2 us; 16384 rows: 99, 73, 75 us)
  const long pieces = ceil_div(a.dim, LINE);
  const int v = pieces > 1024 ? 4 : pieces > 512 || a.tokens > SMS ? 2 : 1;
  const int threads = (int)ceil_div(ceil_div(pieces, v), 32) * 32, rows = std::max(1, 256 / threads);
  const dim3 block(threads, rows);
  const long grid = ceil_div(a.tokens, rows);
  const auto kernel = v == 1 ? norm_add_kernel<T, WIDE, 1> : v == 2 ? norm_add_kernel<T, WIDE, 2> : norm_add_kernel<T, WIDE, 4>;
  return launch_dependent(kernel, dim3((unsigned)grid), block, 0, stream, 0, a);
}

template <typename X, typename T>
static lq_status launch_gate(const GatedArgs &a, bool wide, cudaStream_t stream) {
  const long grid = ceil_div((long)a.tokens * a.warps, GATED_THREADS / 32);
  return launch_dependent(wide ? norm_gate_kernel<X, T, true> : norm_gate_kernel<X, T, false>, dim3((unsigned)grid), dim3(GATED_THREADS), 0, stream, 0, a);
}
template <typename X>
static lq_status launch_gate(const GatedArgs &a, int type, bool wide, cudaStream_t stream) {
  if (type == LQ_F32) return launch_gate<X, float>(a, wide, stream);
  if (type == LQ_F16) return launch_gate<X, __half>(a, wide, stream);
  return launch_gate<X, __nv_bfloat16>(a, wide, stream);
}

// ---- products ----

constexpr int MOST_CHANNELS = 1 << 20;

// [planes][rows][channels] bytes, copied in boxes of `box` rows of `width` (128 or 64) bytes of one plane, swizzled by as many
static bool byte_map(CUtensorMap *map, const void *base, long channels, long rows, long planes, int64_t stride, int64_t plane, int box, int width = PB) {
  const cuuint64_t size[3] = {(cuuint64_t)channels, (cuuint64_t)rows, (cuuint64_t)planes}, strides[2] = {(cuuint64_t)stride, (cuuint64_t)plane};
  const cuuint32_t shape[3] = {(cuuint32_t)width, (cuuint32_t)box, 1}, one[3] = {1, 1, 1};
  const EncodeTiled f = encode_tiled();
  return f && f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(base), size, strides, shape, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                width == PB ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename K>
static lq_status give_shared(K kernel, size_t bytes, std::atomic<uint64_t> &ready) {   // ready: devices on which the kernel has its shared memory
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return LQ_ERR_CUDA;
  const uint64_t bit = uint64_t(1) << (device & 63);
  if (ready.load(std::memory_order_relaxed) & bit) return LQ_OK;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) {
    cudaGetLastError();
    return LQ_ERR_CUDA;
  }
  ready.fetch_or(bit, std::memory_order_relaxed);
  return LQ_OK;
}

template <typename T, bool WIDE, int ROWS>
static lq_status launch_few_t(const ProductMaps &maps, const ProductArgs &a, int grid, cudaStream_t stream) {
  static std::atomic<uint64_t> ready{0};
  const lq_status rc = give_shared(product_few_kernel<T, WIDE, ROWS>, sizeof(FewShared<ROWS>), ready);
  if (rc != LQ_OK) return rc;
  return launch_dependent(product_few_kernel<T, WIDE, ROWS>, dim3(grid), dim3(FEW_THREADS), sizeof(FewShared<ROWS>), stream, a.split, maps, a);
}
// Which kernel: the one whose tiles take fewer rounds over the GPU, as a round of either takes the same time (32 K blocks: 14 - 18 us; 148 tiles of 128 x 128,
// or 74 pairs of CTAs on 256 x 256), the one for few rows where they tie.  Few and many, us: 1024 rows x 4096 x 4096: 2 rounds 30.8, 1 round 17.7; 192 x 4096 x 12352: 2
// rounds 30.2, 1 round 17.7; 512 x 8192 x 1024: a quarter of a round 14.2, 1 round 28.2; 779 x 1296 x 1999, 1 round each: 11.2 and 10.6.
// How many rows a group has is known on the device only: half a tile of every group is taken to be empty.  64 groups x 2048 x 1536 of 64 rows each 47 and 54 us, of 128
// rows 54 and 57 (which the rule gives away), of 192 rows 90 and 60.  What it costs where the rows lie unevenly: 4096 rows of 128 groups, on average 32 (tiles of 32 rows;
// others at best), evenly 71 us (71), all in one group 41 (23); 8192 rows, on average 64 (tiles of 128 rows), evenly 84 (84), all in one 53 (31), half of them in one 67 (66).
static bool are_few(const lq_linear *s, bool grouped, int split) {
  const long few = ceil_div(s->out, PB), many = ceil_div(s->out, MANY_OUTS);
  if (grouped) {
    const double rows = (double)s->rows / s->groups;
    return few * (rows / FEW_ROWS + 0.5) / SMS <= many * std::max(1.0, rows / MANY_ROWS + 0.5) / (SMS / 2);
  }
  return split > 1 || ceil_div(few * ceil_div(s->rows, FEW_ROWS), SMS) <= ceil_div(many * ceil_div(s->rows, MANY_ROWS), SMS / 2);
}
// Few rows: CTAs that share a tile's K blocks.  One row of 4096 x 4096 (32 tiles), weights from memory: 1, 2, 4 CTAs 11.7, 8.6, 7.0 us.  As many as 148 places have room
// for, also where two CTAs with tiles of 32 rows fit an SM: one row of 4096 x 8192 (64 tiles) with two 10.3, with four 9.4; 16 x 12352 x 4096 with four 13.6, eight 12.8;
// but 4096 x 12352 (97 tiles) alone 13.4, with two 14.6, and 64 x 4096 x 4096 (tiles of 128 rows) with four 9.5, six 17.0.
static int split_of(const lq_linear *s, bool grouped, int rows) {
  const long tiles = ceil_div(s->rows, rows) * ceil_div(s->out, PB), blocks = ceil_div(s->in, PB);
  return grouped ? 1 : (int)std::max(1l, std::min({SMS / tiles, 8l, blocks / 2}));
}
template <int ROWS>
static lq_status launch_few(const lq_linear *s, ProductArgs a, const void *x, int64_t x_stride, const void *w, cudaStream_t stream) {
  a.tiles_n = (int)ceil_div(s->out, PB);
  a.tiles_m.set((uint32_t)ceil_div(s->rows, ROWS));
  a.share = a.blocks / a.split, a.more = a.blocks % a.split;
  ProductMaps maps{};
  if ((ROWS > FEW_BOX && !byte_map(&maps.x, x, s->in, s->rows, 1, x_stride, x_stride * s->rows, ROWS)) ||
      !byte_map(&maps.more, x, s->in, s->rows, 1, x_stride, x_stride * s->rows, FEW_BOX) ||
      !byte_map(&maps.w, w, s->in, s->out, s->groups, s->in, (int64_t)s->in * s->out, PB))
    return LQ_ERR_CUDA;
  const long tiles = (ceil_div(s->rows, ROWS) + s->groups - 1) * a.tiles_n;   // at most
  const int grid = (int)std::min<long>(tiles, ROWS == FEW_ROWS ? SMS : 2 * SMS) * a.split;
  const bool wide = aligned(a.out, 16) && a.out_stride % (16 / type_size(s->type)) == 0;
  if (s->type == LQ_F32) return wide ? launch_few_t<float, true, ROWS>(maps, a, grid, stream) : launch_few_t<float, false, ROWS>(maps, a, grid, stream);
  if (s->type == LQ_F16) return wide ? launch_few_t<__half, true, ROWS>(maps, a, grid, stream) : launch_few_t<__half, false, ROWS>(maps, a, grid, stream);
  return wide ? launch_few_t<__nv_bfloat16, true, ROWS>(maps, a, grid, stream) : launch_few_t<__nv_bfloat16, false, ROWS>(maps, a, grid, stream);
}

template <typename T, bool WIDE>
static lq_status launch_many_t(const ProductMaps &maps, const ProductArgs &a, long pairs, cudaStream_t stream) {
  static std::atomic<uint64_t> ready{0};
  const lq_status rc = give_shared(product_many_kernel<T, WIDE>, sizeof(ManyShared), ready);
  if (rc != LQ_OK) return rc;
  return launch_dependent(product_many_kernel<T, WIDE>, dim3(2 * (unsigned)std::min<long>(pairs, SMS / 2)), dim3(MANY_THREADS), sizeof(ManyShared), stream, 0, maps, a);
}
static lq_status launch_many(const lq_linear *s, ProductArgs a, const void *x, int64_t x_stride, const void *w, cudaStream_t stream) {
  a.tiles_n = (int)ceil_div(s->out, MANY_OUTS);
  a.tiles_m.set((uint32_t)ceil_div(s->rows, MANY_ROWS));
  ProductMaps maps{};
  if (!byte_map(&maps.x, x, s->in, s->rows, 1, x_stride, x_stride * s->rows, 128) ||
      !byte_map(&maps.w, w, s->in, s->out, s->groups, s->in, (int64_t)s->in * s->out, 128))
    return LQ_ERR_CUDA;
  const long pairs = (ceil_div(s->rows, MANY_ROWS) + s->groups - 1) * a.tiles_n;   // at most
  const unsigned size = type_size(s->type);
  const bool wide = aligned(a.out, 16) && a.out_stride % (16 / size) == 0 && a.out_stride * size * s->rows < (int64_t)1 << 40;   // (what a tensor map can say)
  if (wide && !byte_map(&maps.more, a.out, (long)s->out * size, s->rows, 1, a.out_stride * size, a.out_stride * size * s->rows, 32, 64)) return LQ_ERR_CUDA;
  if (s->type == LQ_F32) return wide ? launch_many_t<float, true>(maps, a, pairs, stream) : launch_many_t<float, false>(maps, a, pairs, stream);
  if (s->type == LQ_F16) return wide ? launch_many_t<__half, true>(maps, a, pairs, stream) : launch_many_t<__half, false>(maps, a, pairs, stream);
  return wide ? launch_many_t<__nv_bfloat16, true>(maps, a, pairs, stream) : launch_many_t<__nv_bfloat16, false>(maps, a, pairs, stream);
}

static lq_status product(const lq_linear *s, const lq_product_io *io, bool grouped, lq_stream stream) {
  lq_status rc;
  if (!s || !io) return LQ_ERR_NULL;
  if (bad_count(s->rows) || s->in <= 0 || s->out <= 0 || s->groups <= 0 || s->type < LQ_BF16 || s->type > LQ_F32) return LQ_ERR_SHAPE;
  if (!grouped && s->groups != 1) return LQ_ERR_SHAPE;
  if (s->in % 16 != 0 || s->in > MOST_CHANNELS || s->out > MOST_CHANNELS || s->groups > MOST_GROUPS || s->rows > MOST_ROWS) return LQ_ERR_UNSUPPORTED;
  if ((ceil_div(s->rows, FEW_BOX) + s->groups) * ceil_div(s->out, PB) > INT32_MAX - 1024) return LQ_ERR_UNSUPPORTED;   // tiles
  if ((int64_t)s->in * s->out >= (int64_t)1 << 40) return LQ_ERR_UNSUPPORTED;   // (what a tensor map can say)
  if (s->rows == 0) return LQ_OK;
  const uint8_t *x = io->x, *w = io->w;
  const float *x_scale = io->x_scale, *w_scale = io->w_scale;
  void *out = io->out;
  const int64_t x_stride = io->x_stride, x_scale_stride = io->x_scale_stride, out_stride = io->out_stride;
  const int32_t *group_start = grouped ? io->group_start : nullptr;
  if ((rc = check_arrays(16, {x, w})) != LQ_OK) return rc;
  if ((rc = check_arrays(4, {x_scale, w_scale})) != LQ_OK) return rc;
  if ((rc = check_arrays(type_size(s->type), {out})) != LQ_OK) return rc;
  if (grouped && !group_start) return LQ_ERR_NULL;
  if (!aligned(group_start, 4)) return LQ_ERR_ALIGN;
  if (x_stride < s->in || x_scale_stride < s->rows || out_stride < s->out) return LQ_ERR_SHAPE;
  if (x_stride % 16 != 0) return LQ_ERR_ALIGN;
  if (x_stride > (int64_t)1 << 32 || x_stride * s->rows >= (int64_t)1 << 40) return LQ_ERR_UNSUPPORTED;   // (what a tensor map can say)
  const unsigned size = type_size(s->type);
  const int blocks = (int)ceil_div(s->in, PB);
  const Span o{out, out_stride, s->out, s->rows, size};
  for (const Span &in : {Span{x, x_stride, s->in, s->rows, 1}, Span{x_scale, x_scale_stride, s->rows, blocks, 4},
                         Span{w, s->in, s->in, (long)s->out * s->groups, 1}, Span{w_scale, blocks, blocks, ceil_div(s->out, PB) * s->groups, 4},
                         Span{group_start, s->groups + 1, s->groups + 1, 1, 4}})
    if (spans_meet(o, in)) return LQ_ERR_UNSUPPORTED;
  ProductArgs a{x_scale, w_scale, out, x_scale_stride, out_stride, group_start, s->rows, blocks, s->out, s->groups, 0, 1, blocks, 0, {}};
  if (s->rows <= FEW_BOX * (grouped ? s->groups : 1)) {
    a.split = split_of(s, grouped, FEW_BOX);
    return launch_few<FEW_BOX>(s, a, x, x_stride, w, cuda_stream(stream));
  }
  a.split = split_of(s, grouped, FEW_ROWS);
  if (!are_few(s, grouped, a.split)) return launch_many(s, a, x, x_stride, w, cuda_stream(stream));
  return launch_few<FEW_ROWS>(s, a, x, x_stride, w, cuda_stream(stream));
}

// lq_check_device / lq_clear_device_flags: the flag of the kernels in this file
bool linear_flags(int *flags) { return cudaMemcpyFromSymbol(flags, g_product_error, sizeof(int)) == cudaSuccess; }
bool clear_linear_flags() {
  const int zero = 0;
  return cudaMemcpyToSymbol(g_product_error, &zero, sizeof(int)) == cudaSuccess;
}

}  // namespace lq

using namespace lq;

extern "C" {

lq_status lq_norm_add(const lq_add *s, const lq_norm_io *n, lq_stream stream) {
  if (!s || !n) return LQ_ERR_NULL;
  if (bad_count(s->tokens) || s->dim <= 0 || s->norm < LQ_NORM_NONE || s->norm > LQ_NORM_RMS || s->type < LQ_BF16 || s->type > LQ_F32) return LQ_ERR_SHAPE;
  if (s->dim > LQ_NORM_ADD_MOST || s->tokens > MOST_ROWS) return LQ_ERR_UNSUPPORTED;
  if (s->tokens == 0) return LQ_OK;
  const unsigned size = type_size(s->type);
  const NormIo io{{n->x, n->residual}, {n->x_stride, n->residual_stride}, {size, size}, true, n->w, s->norm == LQ_NORM_RMS ? s->dim : 0, norm_out(n)};
  const lq_status rc = check_norm_io(io, s->tokens, s->dim, s->type, true);
  if (rc != LQ_OK) return rc;
  const AddArgs a{n->x, n->residual, n->w, n->x_stride, n->residual_stride, io.o, s->tokens, s->dim, s->norm, s->eps, s->norm == LQ_NORM_RMS ? 1.0f / s->dim : 1.0f};
  const bool wide = wide_norm(io, s->dim, s->type, LINE);
  if (s->type == LQ_F32) return wide ? launch_add<float, true>(a, cuda_stream(stream)) : launch_add<float, false>(a, cuda_stream(stream));
  if (s->type == LQ_F16) return wide ? launch_add<__half, true>(a, cuda_stream(stream)) : launch_add<__half, false>(a, cuda_stream(stream));
  return wide ? launch_add<__nv_bfloat16, true>(a, cuda_stream(stream)) : launch_add<__nv_bfloat16, false>(a, cuda_stream(stream));
}

lq_status lq_norm_gate(const lq_gated *s, const lq_norm_io *n, lq_stream stream) {
  if (!s || !n) return LQ_ERR_NULL;
  if (bad_count(s->tokens) || s->heads <= 0 || s->dim <= 0 || s->norm < LQ_NORM_NONE || s->norm > LQ_NORM_RMS) return LQ_ERR_SHAPE;
  if ((s->silu != 0 && s->silu != 1) || s->type < LQ_BF16 || s->type > LQ_F32 || s->o_type < LQ_BF16 || s->o_type > LQ_F32) return LQ_ERR_SHAPE;
  const long warps = ceil_div((long)s->heads * s->dim, 32 * GATED_LINE);
  if ((s->dim != 64 && s->dim != 128 && s->dim != 256) || s->heads > (1 << 16) || warps * s->tokens > MOST_ROWS) return LQ_ERR_UNSUPPORTED;
  if (s->tokens == 0) return LQ_OK;
  if (!n->z) return LQ_ERR_NULL;
  const long width = (long)s->heads * s->dim;
  const NormIo io{{n->x, n->z}, {n->x_stride, n->z_stride}, {type_size(s->o_type), type_size(s->type)}, false, n->w, s->norm == LQ_NORM_RMS ? s->dim : 0, norm_out(n)};
  const lq_status rc = check_norm_io(io, s->tokens, width, s->type, false);
  if (rc != LQ_OK) return rc;
  GatedArgs a{n->x, n->z, n->w, n->x_stride, n->z_stride, io.o, s->tokens, s->heads, s->dim, s->norm, s->silu, s->eps, s->norm == LQ_NORM_RMS ? 1.0f / s->dim : 1.0f, (int)warps, {}};
  a.by_warps.set((uint32_t)warps);
  const bool wide = wide_norm(io, width, s->type, GATED_LINE);
  if (s->o_type == LQ_F32) return launch_gate<float>(a, s->type, wide, cuda_stream(stream));
  if (s->o_type == LQ_F16) return launch_gate<__half>(a, s->type, wide, cuda_stream(stream));
  return launch_gate<__nv_bfloat16>(a, s->type, wide, cuda_stream(stream));
}

lq_status lq_product(const lq_linear *shape, const lq_product_io *io, lq_stream stream) { return product(shape, io, false, stream); }

lq_status lq_product_groups(const lq_linear *shape, const lq_product_io *io, lq_stream stream) { return product(shape, io, true, stream); }

}  // extern "C"
