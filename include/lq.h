/*
 * lq.h - C boundary of the B200 (sm_100a) per-window 8-bit decode step for
 * Gated DeltaNet (scalar gate) and Kimi Delta Attention (per-channel gate)
 * recurrent states.
 *
 * One value head owns a state S in R^{d_k x d_v} (Sec. 3.1, Eq. 1; row index =
 * key channel, column index = value channel, readout o = S^T q).  Between
 * window boundaries the state is held as
 *     S_l = Gamma_{1:l} [ C (Z/127) B + Kc Uc^T ] + sum_j Gamma_{j+1:l} kt_j u_j^T      (Eq. 7)
 * with Z the 8-bit codes, B the per-value-channel scale, C = Diag(c) the
 * per-key-row smoothing scale (Sec. 3.4), (Kc, Uc) the r fp16 Compensator
 * Tokens (Sec. 3.3) and (alpha_j, kt_j, u_j) the buffered records of the
 * tokens decoded since the boundary (Sec. 3.2, Eq. 3).
 *
 * Conventions for every entry point
 *  - All pointers are DEVICE pointers owned by the caller unless a parameter
 *    is documented as a host pointer.  Arrays are dense, row-major, in the
 *    layouts given below, and must be 16-byte aligned.
 *  - The library allocates no device memory and never synchronises: work is
 *    enqueued on `stream` and the call returns.  The lq_shape and lq_state
 *    structs themselves are read on the host during the call only.
 *  - bf16 and fp16 values travel as their 16-bit patterns (uint16_t).
 *  - Errors are reported through the return value; nothing aborts or throws.
 *    Argument errors are detected before anything is enqueued (the host-buffer
 *    entry points included).
 *  - Arithmetic is IEEE binary32.  Sums over a channel index are taken in a
 *    fixed order (blocks of eight consecutive terms; inside a block the
 *    even-numbered and the odd-numbered terms are two chains of fused
 *    multiply-adds that are added at the end; block results combined as a
 *    balanced binary tree over the block index, neighbours first), and the
 *    code-matrix term of the readout is an exact integer sum, so results do
 *    not depend on the launch configuration and are reproducible bit for bit.
 *  - Supported shapes: d_k = d_v = 128, 1 <= W <= 64, 0 <= r <= 16,
 *    n_iter >= 1, heads_v a multiple of heads_qk.  Anything else returns
 *    LQ_ERR_UNSUPPORTED.
 */
#ifndef LQ_H_
#define LQ_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LQ_OK = 0,
  LQ_ERR_NULL = 1,        /* a required pointer is null                         */
  LQ_ERR_SHAPE = 2,       /* a dimension is non-positive or inconsistent        */
  LQ_ERR_ALIGN = 3,       /* a pointer is not 16-byte aligned                   */
  LQ_ERR_UNSUPPORTED = 4, /* valid request outside the supported shapes         */
  LQ_ERR_CUDA = 5,        /* the CUDA runtime reported an error on launch/copy  */
  LQ_ERR_TOO_LARGE = 6    /* the request does not fit the library's built-in scratch buffer */
} lq_status;

typedef enum {
  LQ_GATE_SCALAR = 0, /* GDN: D_t = alpha_t I;       alpha is [B,Hv]       */
  LQ_GATE_DIAG = 1    /* KDA: D_t = Diag(alpha_t);   alpha is [B,Hv,d_k]   */
} lq_gate;

/* CUDA stream handle (a cudaStream_t); null is the default stream. */
typedef struct CUstream_st *lq_stream;

typedef struct {
  int batch;    /* B: sequences                                                   */
  int heads_v;  /* Hv: value heads per sequence, one state each                   */
  int heads_qk; /* Hqk: query/key heads; value head h reads q/k head h/(Hv/Hqk)   */
  int d_k, d_v; /* state is d_k x d_v                                             */
  int W;        /* window length (the paper's p)                                  */
  int r;        /* Compensator Tokens per state                                   */
  int n_iter;   /* rounds of the power iteration at a boundary (1 is the default of */
                /* the binding).  All r vectors are iterated together: T = S W,     */
                /* orthonormalise, W = S^T T, orthonormalise, ...; column h of W    */
                /* starts from the u of the (h+1)-th newest buffered record, or     */
                /* from Walsh function h where there is no such record              */
  int gate;     /* lq_gate                                                        */
  int smooth;   /* 1: residual smoothing (Sec. 3.4); 0: c = 1 (ablation)          */
  int delta;    /* 1: delta rule, the correction reads the state back with          */
                /* b = alpha (.) k (DeltaNet, Gated DeltaNet, KDA);                 */
                /* 0: b = 0, u = v (the other instances of the paper's Table 4:     */
                /* linear attention, RetNet, Mamba2 with the scalar gate; GLA,      */
                /* RWKV6, HGRN2 with the diagonal gate; pass beta = 1 for k~ = k)   */
  int rec16;    /* 1: the record buffer holds fp16 values, as in the paper's storage      */
                /* accounting (kt, u and the diagonal gate's alpha are rounded, with       */
                /* saturation, when a record is appended; the scalar gate's decays stay    */
                /* fp32; `o` of the appending token uses the unrounded u); 0: fp32 records */
  int state_bf16; /* 1: "per-window BF16", the -w baseline of the paper's Fig. 3 and Table 2: the    */
                /* boundary state is the dense state rounded to bfloat16 (nearest even) once per  */
                /* window, with no scale, smoothing or compensator; needs r = 0 and smooth = 0;   */
                /* the readout is S0^T x in binary32 in the fixed summation order.  0: the 8-bit  */
                /* representation of Eq. 7                                                        */
} lq_shape;

/*
 * Window representation of B x Hv states, laid out for bulk transfers: everything that is read once per
 * token and head is contiguous.
 *
 * heads: one block of lq_head_bytes(shape) bytes per (sequence, value head), [B,Hv] blocks back to back:
 *     offset 0                        codes      int8 [d_v][d_k]  Z^T: the code of S[i][j] sits at [j][i]
 *                                                (value-channel major, so that the key index is contiguous);
 *                                                symmetric, in [-127,127]
 *     + d_k*d_v                       col_scale  fp32 [d_v]       step of the code per value channel, B_j/127:
 *                                                dequant(Z)_ij = Z_ij * col_scale_j  (Appendix B.3)
 *     + 4*d_v                         row_smooth fp32 [d_k]       c > 0 (Sec. 3.4)
 *     + 4*d_k                         comp_k     fp16 [r][d_k]    unit-length key side of the compensators
 *     + 2*r*d_k                       comp_u     fp16 [r][d_v]    value side (carries the magnitude)
 *   (17408 + 512 r bytes at d_k = d_v = 128: 19456 for r = 4, i.e. 1.19 bytes per state element.)
 *   With shape.state_bf16 the block is instead   state  bf16 [d_v][d_k]   S0^T: S0[i][j] sits at [j][i]
 *   (32768 bytes).
 *
 * records: one row of lq_record_floats(shape) values (fp32, or fp16 with shape.rec16) per buffered record, [B,Hv,W] rows:
 *     kt[d_k] | u[d_v]                write key kt = beta*k and correction u = v - S^T(alpha.k)  (Eq. 3)
 *     | alpha[d_k]                    diagonal gate only: the record's decay
 * decays: scalar gate only, fp32 [B,Hv,W]: the decay of each buffered record (ignored for the diagonal gate).
 * win_pos: int32 [B], records buffered per sequence, 0..W-1 between calls.  Bits 16 and up are used as a
 *     scratch counter while a call runs and are zero again when it has finished.
 * work: optional (may be null): int32 [LQ_WORK_WORDS], all zero when the state is created and zero again after
 *     every call.  With it, lq_decode_step takes tokens and window boundaries of many shapes in one launch instead
 *     of two, and the decode kernel of the others hands out the heads of its last, partial round (B*Hv heads over
 *     the CTAs that are resident at once) to the CTAs that get there first, instead of giving every CTA the same
 *     number of heads: on a GPU whose memory system does not serve all SMs alike, equal shares do not take equal
 *     time.  Results are the same bit for bit either way.  Sub-batches of one state that are
 *     addressed by pointer offset may share one `work` as long as their calls do not run at the same time (calls
 *     in one stream never do).  After a call that returned LQ_ERR_CUDA the words are to be zeroed again (and the
 *     state restored from a checkpoint: a step that was enqueued in part leaves neither valid).
 */
#define LQ_WORK_WORDS 8
typedef struct {
  uint8_t *heads;
  void *records;   /* float rows, or (shape.rec16) fp16 rows of the same element counts */
  float *decays;
  int32_t *win_pos;
  int32_t *work;
} lq_state;

/* Size in bytes of one head block, and the number of fp32 values in one record row (0 for an invalid shape). */
uint64_t lq_head_bytes(const lq_shape *shape);
uint64_t lq_record_floats(const lq_shape *shape);

/*
 * One decode token for every (sequence, value head): Eq. 10 (the readout of the smoothed, compensated
 * window representation) applied to alpha.k gives the correction u of Eq. 3, applied to alpha.q gives
 * the output through S_l^T q = S_{l-1}^T (alpha.q) + u (kt^T q); the record (alpha, kt, u) is appended
 * to the buffer and win_pos advances.  A sequence whose window becomes full (win_pos reaches W) is
 * taken through the boundary in the same call, as Eq. 4 prescribes: see lq_window_flush.
 *   q, k  : bf16 [B,Hqk,d_k]     v : bf16 [B,Hv,d_v]     beta : bf16 [B,Hv]
 *   alpha : bf16 [B,Hv] or [B,Hv,d_k], the decay multiplier itself (not its logarithm)
 *   o     : fp32 [B,Hv,d_v], written
 * A sequence that enters with win_pos >= W (possible only if the caller set it) gets no token: its `o`
 * rows are not written and nothing is appended; with win_pos == W it is taken through the boundary by
 * this call like by lq_window_flush.
 * Calls on the same state must be ordered by the stream.
 */
lq_status lq_decode_step(const lq_shape *shape, const lq_state *state, const uint16_t *q, const uint16_t *k,
                         const uint16_t *v, const uint16_t *beta, const uint16_t *alpha, float *o, lq_stream stream);

/*
 * lq_decode_step for a measuring harness: the same results, and in addition the CUDA event `event_between`
 * (a cudaEvent_t created by the caller; may be null) is recorded on `stream` between the decode kernel and
 * the window-boundary kernel, so that the two can be timed separately.  With an event the step is always these
 * two launches, also where lq_decode_step makes one of both (lq_step_launches).
 */
lq_status lq_decode_step_profiled(const lq_shape *shape, const lq_state *state, const uint16_t *q, const uint16_t *k,
                                  const uint16_t *v, const uint16_t *beta, const uint16_t *alpha, float *o,
                                  lq_stream stream, void *event_between);

/*
 * Same as lq_decode_step, but the token's inputs and the output live in HOST memory (pinned memory makes
 * the copies asynchronous): q_h, k_h, v_h, beta_h, alpha_h are copied into the device staging buffer
 * `stage` on `stream`, the step runs, and `o` is copied to o_h.  `stage` is a device buffer of at least
 * lq_decode_stage_bytes(shape) bytes, 16-byte aligned, owned by the caller.  The host arrays must stay
 * valid until the stream has passed the call.
 */
lq_status lq_decode_step_host(const lq_shape *shape, const lq_state *state, const uint16_t *q_h,
                              const uint16_t *k_h, const uint16_t *v_h, const uint16_t *beta_h,
                              const uint16_t *alpha_h, float *o_h, void *stage, lq_stream stream);
/*
 * lq_decode_step_host with the host<->device transfers overlapped with the kernels.  (The paper's path
 * starts and ends in device memory; this is a convenience of the library for callers whose tokens arrive in
 * host memory.)  The batch is cut into two sub-batches of whole sequences.  The inputs of both are brought in
 * on a copy-in stream, so the second sub-batch arrives while the first is computed; o of a sub-batch is
 * complete after its decode kernel and is copied out on a copy-out stream while the next sub-batch and the window
 * boundaries (one launch for the whole batch) run.  The two side streams are created per device at the first call
 * (make that call outside any stream capture) and are tied to `stream` by events on both sides: the call
 * starts after everything already enqueued on `stream`, and anything enqueued on `stream` afterwards starts
 * after the last copy.  Same arguments, staging size, results and error codes as lq_decode_step_host; use
 * pinned host memory, otherwise nothing overlaps.  Batches below sixteen sequences take the unpipelined path.
 * Calls from several host threads are serialised inside the library while they enqueue.
 *
 * Consecutive calls with the same `stage`, `stream` and shape chain onto each other: the inputs of sub-batch c of
 * the later call are brought in as soon as the earlier call's decode kernel of sub-batch c has consumed its own,
 * i.e. next to the earlier call's window-boundary kernels and copies out, and possibly before other work that
 * was enqueued on `stream` in between.  So the host input arrays must hold their final values when the call is
 * made (not merely when `stream` reaches it), and between such calls `stage` belongs to the library.  A call of
 * lq_decode_step_host or lq_decode_step_host_static, another `stage` or another stream ends the chain; the next
 * pipelined call is then ordered after everything on `stream` again.  Outputs are always stream-ordered: what is
 * enqueued on `stream` after a call finds o_h complete.
 *
 * Both host-buffer entry points read the inputs with ONE gather launch (per sub-batch) instead of five copies
 * when all input arrays are pinned, mapped into the device (cudaHostAlloc / cudaHostRegister memory under
 * unified addressing) and 16-byte aligned with sizes that are multiples of 16 bytes; lq_decode_step_host
 * then also lets the decode kernel write o straight into the host array.  Otherwise they fall back to
 * cudaMemcpyAsync.  The results are the same either way.
 */
lq_status lq_decode_step_host_pipelined(const lq_shape *shape, const lq_state *state, const uint16_t *q_h,
                                        const uint16_t *k_h, const uint16_t *v_h, const uint16_t *beta_h,
                                        const uint16_t *alpha_h, float *o_h, void *stage, lq_stream stream);
/* Bytes of device staging lq_decode_step_host needs for `shape` (0 if the shape is invalid). */
uint64_t lq_decode_stage_bytes(const lq_shape *shape);

/*
 * lq_decode_step_host for callers that cannot hand over a staging buffer because they cannot allocate one.
 * (The paper has no counterpart: this is a convenience of the library.)
 *
 * Who this is for: a serving process that gave all of the device's memory to its own pools when it started
 * has nothing left for cudaMalloc to return, and a decode loop that must never stall cannot afford
 * cudaMalloc/cudaFree either, since both may synchronise the whole device.  Such a caller still owns the
 * host arrays and the lq_state, but has nowhere to put the few megabytes of staging that the host-buffer
 * path needs.  Here the staging lives inside the library, in a fixed device array of
 * LQ_STATIC_STAGE_BYTES bytes that every GPU that loads the library keeps reserved until the process
 * exits.  The call itself allocates and frees nothing, on the device or through any library.
 *
 * Same arguments and behaviour as lq_decode_step_host without `stage`, with these differences:
 *  - lq_decode_stage_bytes(shape) must not exceed LQ_STATIC_STAGE_BYTES, otherwise LQ_ERR_TOO_LARGE is
 *    returned and nothing is enqueued (16 MiB covers 256 sequences x 32 heads, the benchmark batch).
 *  - The first call on each device looks up the device address of the built-in array (with that device
 *    current).  Make that first call outside any stream capture.
 *  - The array is shared by all calls and keeps what the previous call left in it.  The output staging is
 *    therefore cleared at the start of every call: rows of o_h that belong to sequences which get no token
 *    (win_pos >= W on entry) come back as zeros.
 *  - Because the array is shared, two calls whose work overlaps on the GPU (different streams, or different
 *    host threads) race on it.  Order them on one stream, or use lq_decode_step_host with separate buffers.
 */
#define LQ_STATIC_STAGE_BYTES (16u << 20)
lq_status lq_decode_step_host_static(const lq_shape *shape, const lq_state *state, const uint16_t *q_h,
                                     const uint16_t *k_h, const uint16_t *v_h, const uint16_t *beta_h,
                                     const uint16_t *alpha_h, float *o_h, lq_stream stream);

/*
 * Window boundary (Secs. 3.2-3.4): for every sequence with win_pos == W, or, when force != 0, with
 * win_pos > 0, rebuild the dense state from the window representation (Eq. 7), refit the r Compensator
 * Tokens by power iteration and remove them (Eqs. 5-6), recompute the smoothing scales from the
 * residual, requantize it to 8 bits, and set win_pos = 0.  Other sequences are not touched.
 */
lq_status lq_window_flush(const lq_shape *shape, const lq_state *state, int force, lq_stream stream);

/*
 * Start a window from dense states: S fp32 [B,Hv,d_k,d_v] (read only) is split into compensators,
 * smoothing scales and 8-bit codes exactly as at a window boundary; win_pos is set to 0 for all B
 * sequences.  The record buffers are not read or written.
 */
lq_status lq_quantize_state(const lq_shape *shape, const float *S, const lq_state *state, lq_stream stream);

/*
 * The dense state the window representation currently stands for, all buffered records applied (Eq. 7
 * with l = win_pos): written to S fp32 [B,Hv,d_k,d_v].  The state is not modified.
 */
lq_status lq_dequantize_state(const lq_shape *shape, const lq_state *state, float *S, lq_stream stream);

/*
 * The window representation as separate arrays in the paper's notation and orientation (Sec. 3.1: S is d_k x d_v;
 * Appendix B.3 for Z and B; Sec. 3.4 for c; Sec. 3.3 for the compensators; Eq. 3 for the records), for callers
 * that hold or want the state that way instead of in the packed head blocks above.  All arrays dense, row-major,
 * device memory, 16-byte aligned:
 *   codes      int8 [B,Hv,d_k,d_v]   Z (NOT transposed)
 *   col_scale  fp32 [B,Hv,d_v]       step of the code per value channel, B_j / 127
 *   row_smooth fp32 [B,Hv,d_k]       c
 *   comp_k     fp16 [B,Hv,r,d_k]     comp_u  fp16 [B,Hv,r,d_v]      (null when r = 0)
 *   buf_k      fp32 [B,Hv,W,d_k]     write keys beta*k of the buffered records
 *   buf_u      fp32 [B,Hv,W,d_v]     corrections u
 *   buf_a      fp32 [B,Hv,W] (scalar gate) or [B,Hv,W,d_k] (diagonal gate): the records' decays
 *   win_pos    int32 [B]
 * lq_import_state fills `dst` from the arrays, lq_export_state the arrays from `src`; both copy all W record
 * slots whatever win_pos says.  With shape.rec16 the records are narrowed to fp16 on import (nearest even,
 * saturating) and widened on export.  Not available with shape.state_bf16 (LQ_ERR_UNSUPPORTED).
 */
typedef struct {
  int8_t *codes;
  float *col_scale;
  float *row_smooth;
  uint16_t *comp_k;
  uint16_t *comp_u;
  float *buf_k;
  float *buf_u;
  float *buf_a;
  int32_t *win_pos;
} lq_state_arrays;
lq_status lq_import_state(const lq_shape *shape, const lq_state_arrays *src, const lq_state *dst, lq_stream stream);
lq_status lq_export_state(const lq_shape *shape, const lq_state *src, const lq_state_arrays *dst, lq_stream stream);

/*
 * Speed and accuracy baselines: the same token on an unquantized dense state (Eq. 1 with the GDN / KDA
 * coefficients of Table 4), read and written in full every token.  S is [B,Hv,d_k,d_v], fp32 or bf16
 * (rounded to nearest even after every token, the "BF16 per-step" setting); o is computed from the
 * updated state before it is rounded.  Only batch, heads_v, heads_qk, d_k, d_v and gate of `shape` are used.
 */
lq_status lq_ref_decode_step_f32(const lq_shape *shape, float *S, const uint16_t *q, const uint16_t *k,
                                 const uint16_t *v, const uint16_t *beta, const uint16_t *alpha, float *o,
                                 lq_stream stream);
lq_status lq_ref_decode_step_bf16(const lq_shape *shape, uint16_t *S, const uint16_t *q, const uint16_t *k,
                                  const uint16_t *v, const uint16_t *beta, const uint16_t *alpha, float *o,
                                  lq_stream stream);

/*
 * ---- What surrounds the decode step in a layer ----------------------------------------------------------------
 *
 * The projections of a layer with a recurrent state go through a short causal convolution, q and k are normalised
 * per head (and rotated, where the layer's instance rotates), and a prompt's tokens are scanned before the first
 * token is decoded:
 *     prompt:  lq_conv_prompt -> lq_norm_rotate -> lq_scan_prompt -> lq_quantize_state
 *     token:   lq_conv_step   -> lq_norm_rotate -> lq_decode_step (or, on the dense state, lq_scan_step)
 * In front of and behind either, from the residual stream and back to it, with activations and weights in 8 bits:
 *     lq_norm_add -> lq_product (projections) -> ... -> lq_norm_gate -> lq_product (output projection) -> lq_norm_add ...
 * The scans are those of the instances with b = 0 and a scalar decay (lq_shape.delta = 0, LQ_GATE_SCALAR).  For the delta rule and for decays per
 * key channel nothing here goes from a prompt to its dense state: lq_quantize_state takes one that the caller has made.
 * lq_decode_step takes dense arrays: slices of rows that lq_conv_step has left are copied in front of it.  It has neither `select` nor `skip`: its beta
 * and alpha are gates, and the skip is added to its o.
 *
 * Conventions of these entry points, next to those at the top of this file:
 *  - Tokens are ROWS.  The rows of the sequences of a call lie back to back: sequence n has rows seq_start[n] to
 *    seq_start[n+1] - 1 (int32 [seqs + 1] in device memory, not decreasing; rows in front of seq_start[0] and from
 *    seq_start[seqs] on belong to nobody: they are not written, and what they hold does not matter).  The single-token forms have one row
 *    per sequence, row n.
 *  - A row's channels are contiguous, `..._stride` is the distance between rows in elements, at least a row long:
 *    slices of a wider projection are taken as they are.  Such arrays need the alignment of their element type only,
 *    except for q, k, v and o of the scan: 16 bytes, and strides that are multiples of 8.  All other arrays are dense.
 *  - States are kept in SLOTS: sequence n has slot slots[n] (int32 [seqs] in device memory; null: slot n).  Where slots[n] is
 *    negative or not below n_slots, the sequence is padding: none of its rows is written and no state is touched.  No two
 *    sequences of a call may share a slot.
 *  - resume (int32 [seqs] in device memory; null: zero): where it is zero the prompt starts from an empty state (what the
 *    slot holds is not read), elsewhere it goes on from what its slot holds.
 *  - Sums are taken in binary32, in an order that depends on the shapes alone:
 *    the same call gives the same bits again.
 *  - Convolution and scan: at most 2^31 - 1024 rows and sequences, scan: seqs * heads_v at most 2^30 (LQ_ERR_UNSUPPORTED beyond).
 */
typedef enum { LQ_BF16 = 0, LQ_F16 = 1, LQ_F32 = 2 } lq_type;

/*
 * Short causal depthwise convolution with an optional bias and SiLU:
 *     out[t][c] = f( bias[c] + sum_{i < width} w[c][i] x[t - (width-1) + i][c] ),    f(y) = y or y / (1 + exp(-y))
 * in binary32, rounded once to `type` (SiLU: within 2^-21 + 2^-23 |y| of itself in front of that, and 0 for y below -87.3, where it is smaller than
 * 2^-119).  Rows in front of the sequence's first are the state's (resumed) or zero.
 *   x, out : [tokens][channels], strided rows     w : [channels][width]     bias : [channels] or null
 *   state  : [n_slots][width-1][channels], the last width-1 rows of x, oldest first, in and out (lq_conv_prompt: null
 *            if the prompts are fresh and no state is wanted)                                          - all of `type`
 * The slot of a sequence without rows is left as it is.
 * lq_conv_step's out may be its x (same pointer and stride).  Otherwise out must not overlap x, nor state either of them:
 * LQ_ERR_UNSUPPORTED where the ranges show that they do.
 */
typedef struct {
  int tokens;   /* rows (lq_conv_step: equal to seqs)  */
  int seqs;
  int channels;
  int width;    /* taps: 2, 3 or 4                      */
  int n_slots;
  int silu;     /* 1: f is SiLU; 0: f is the identity   */
  int type;     /* lq_type of all arrays                */
} lq_conv;
lq_status lq_conv_prompt(const lq_conv *shape, const void *x, int64_t x_stride, const void *w, const void *bias, void *state,
                         void *out, int64_t out_stride, const int32_t *seq_start, const int32_t *slots,
                         const int32_t *resume, lq_stream stream);
lq_status lq_conv_step(const lq_conv *shape, const void *x, int64_t x_stride, const void *w, const void *bias, void *state,
                       void *out, int64_t out_stride, const int32_t *slots, lq_stream stream);

/*
 * Queries and keys of every row normalised per head and rotated by the row's position, in one pass:
 *     y = x                                           (LQ_NORM_NONE)
 *     y = x / sqrt(sum_i x_i^2 + eps)                 (LQ_NORM_L2)
 *     y = x / sqrt(sum_i x_i^2 / dim + eps) * w       (LQ_NORM_RMS; w null: 1)
 *     y = scale * y
 *     (y_a, y_b) <- (y_a cos - y_b sin, y_b cos + y_a sin),  angle = position * inv_freq[i],  i < rot/2,
 * with (a, b) = (i, i + rot/2), or (2i, 2i + 1) with `pairs`; channels from `rot` on are not rotated.  Rounded once to `type`.
 *   q, out_q : [tokens][heads_q][dim]   k, out_k : [tokens][heads_k][dim], strided rows (heads of a row back to back)
 *   w_q, w_k : fp32 [dim] or null       positions : int32 [tokens]      inv_freq : fp32 [rot/2] (positions, inv_freq: null if
 *                                                                        rot = 0)
 * A row with a negative position is padding: it is not written.  An output may be its own input (same pointer and stride);
 * no other overlap is allowed.  The angle is taken modulo one turn in 64 bits, so far positions lose nothing.
 * Channels that a frequency turns which is not finite become NaN.
 * heads_q or heads_k may be zero (its pointers are not looked at then).
 */
enum { LQ_NORM_NONE = 0, LQ_NORM_L2 = 1, LQ_NORM_RMS = 2 };
typedef struct {
  int tokens;
  int heads_q, heads_k;
  int dim;      /* channels of a head: 64, 128 or 256                    */
  int rot;      /* channels that are rotated: 0 .. dim, a multiple of 16 */
  int pairs;    /* 1: neighbouring channels are a pair; 0: i and i + rot/2 */
  int norm;
  int type;     /* lq_type of q, k and the outputs                       */
  float eps;
  float scale_q, scale_k;
} lq_norm;
lq_status lq_norm_rotate(const lq_norm *shape, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                         void *out_q, int64_t out_q_stride, void *out_k, int64_t out_k_stride, const float *w_q,
                         const float *w_k, const int32_t *positions, const float *inv_freq, lq_stream stream);

/*
 * Selective state space scan with a scalar decay per head (the instances with b = 0 of lq_shape.delta: Mamba2, RetNet, linear
 * attention), on dense states:
 *     S_t = alpha_t S_{t-1} + beta_t k_t v_t^T,      o_t = S_t^T q_t + skip v_t
 * Value head h reads q/k head h/(Hv/Hqk), as in lq_decode_step.  With `select`, beta holds the raw step dt and
 *     dt' = log(1 + exp(dt + dt_bias_h)),   beta_t = dt',   alpha_t = exp(dt' A_h)      (alpha is not looked at).
 *   q, k : bf16 [tokens][Hqk][d_k]    v : bf16 [tokens][Hv][d_v]      strided rows, 16-byte aligned, strides multiples of 8 (o too)
 *   beta, alpha : [tokens][Hv] of gate_type, strided rows; alpha in [0, 1]
 *   A, dt_bias, skip : fp32 [Hv]; dt_bias and skip may be null (0); A is needed with `select` only, and is not positive
 *   S : fp32 [n_slots][Hv][d_k][d_v], written - what lq_quantize_state takes - and, where S0 is null, what resumed sequences start from
 *   S0 : fp32, as S, read only: resumed sequences start from here and S0 stays as it is (a kept prefix that several continuations share);
 *       null: from S.  S itself, or without an element in common with it.
 * lq_scan_prompt: o is bf16.  The outputs are rounded to bf16 once; in front of that the state and the weighted scores of a
 * block of tokens are rounded to bf16 where they enter a product, as the inputs are; S is held and updated in binary32.  A product of decays
 * since the start of a block (128 rows) that is below 2^-126 counts as 0 in S, and as 2^-60 where it is below that in the share S^T q of o; where a long
 * prompt of few heads is cut, so does one since the start of a piece in S.  Outputs beyond 2^67 may overflow.
 * A NaN or an infinity in a row makes o undefined from the first row of its block (128 rows from the sequence's first on) to
 * the end of its sequence, and S of that sequence; other sequences never see it.
 * lq_scan_step: one row per sequence (tokens = seqs), every sequence is resumed, o is fp32 [seqs][Hv][d_v] in strided rows.
 * A sequence without rows has the state it starts from in its slot afterwards: what it is resumed from, or zeros.
 * Neither may have S, S0, o and the inputs overlap (but for S0 = S): LQ_ERR_UNSUPPORTED where the ranges of S, S0, o, q, k and v show it.
 *
 * `work`: lq_scan_prompt_bytes(shape) bytes of device memory, 16-byte aligned, for the states between the pieces that long prompts are
 * cut into and for handing out the heads (null if that is 0).  Its contents mean nothing between calls; calls that may run at the same time need one each.
 */
typedef struct {
  int tokens;    /* rows (lq_scan_step: equal to seqs)                                                      */
  int seqs;
  int max_len;   /* lq_scan_prompt: at least the length of the longest sequence; rows of a sequence beyond it are left out */
  int heads_v, heads_qk;
  int d_k, d_v;  /* 128, 128                                                                                */
  int n_slots;
  int select;
  int gate_type; /* lq_type of beta and alpha: LQ_BF16 or LQ_F32                                            */
} lq_scan;
typedef struct {
  const uint16_t *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const void *beta, *alpha;
  int64_t beta_stride, alpha_stride;
  const float *A, *dt_bias, *skip;
  const float *S0;
  float *S;
  const int32_t *seq_start, *slots, *resume;   /* lq_scan_step: seq_start and resume are not looked at */
} lq_scan_io;
uint64_t lq_scan_prompt_bytes(const lq_scan *shape);
lq_status lq_scan_prompt(const lq_scan *shape, const lq_scan_io *io, uint16_t *o, int64_t o_stride, void *work, lq_stream stream);
lq_status lq_scan_step(const lq_scan *shape, const lq_scan_io *io, float *o, int64_t o_stride, lq_stream stream);

/*
 * ---- The 8-bit linear layer: norms that leave e4m3 rows, products that take them -------------------------------
 *
 * A row of e4m3 codes has a scale for every block of 128 consecutive channels (the last block of a row may be shorter):
 *     value = code * scale,     scale = max(max_block |y|, 448 * 2^-100) / 448,     code = y / scale rounded to e4m3 (nearest even)
 * in binary32: the scale is within 2^-23 of that (relative), and what is rounded to e4m3 within 2^-22 of y / scale, so that a value as close as that to
 * the middle between two codes may get either; beyond 448 it is 448.
 * Arrays need the alignment of their elements only, except for x and w of the products.
 * scale lies block by block: fp32 [ceil(channels/128)][scale_stride], the scales of neighbouring rows side by side, scale_stride at least
 * the number of rows.  A block with an infinity stands for NaN throughout, a NaN for itself alone.  Codes are the 8-bit patterns of e4m3
 * (torch.float8_e4m3fn).
 *
 * lq_norm_add: the residual's addition and the norm of whole rows, in one pass:
 *     h = x + residual,  residual <- h,    y = norm(h) * w,     norm: LQ_NORM_NONE, LQ_NORM_L2 or LQ_NORM_RMS over `dim` channels
 * in binary32 (y from h before it is rounded; a row whose sum of squares is beyond binary32 becomes 0); residual and out are rounded to `type` once, out8
 * and scale as above.
 *   x, out, residual : [tokens][dim] of `type`, strided rows; residual null: h = x.  out may be x (same pointer and stride)
 *   out8             : e4m3 [tokens][dim], strided rows, with `scale`.  Either out or out8 may be null
 *   w                : fp32 [dim] or null (1; LQ_NORM_RMS only)
 * Apart from that no output (residual is one) may overlap an input or another output.
 * dim at most LQ_NORM_ADD_MOST.  With LQ_NORM_NONE and no residual it turns rows of any origin into 8-bit ones.
 */
#define LQ_NORM_ADD_MOST 16384
typedef struct {
  int tokens;
  int dim;
  int norm;
  int type;    /* lq_type of x, residual and out */
  float eps;
} lq_add;
typedef struct {
  const void *x;         /* lq_norm_gate: o              */
  int64_t x_stride;
  void *residual;        /* lq_norm_add, in and out      */
  int64_t residual_stride;
  const void *z;         /* lq_norm_gate                 */
  int64_t z_stride;
  const float *w;
  void *out;
  int64_t out_stride;
  uint8_t *out8;
  int64_t out8_stride;
  float *scale;          /* where out8 is not null       */
  int64_t scale_stride;
} lq_norm_io;            /* what a form does not have is not looked at */
lq_status lq_norm_add(const lq_add *shape, const lq_norm_io *io, lq_stream stream);

/*
 * lq_norm_gate: the outputs of the recurrence normalised per head, weighted and gated:
 *     y = norm(o) * w * f(z),     f(z) = z / (1 + exp(-z)) (silu) or 1 / (1 + exp(-z))
 * in binary32 (f: within 2^-21 + 2^-23 |z| of itself, relative, with LQ_F32 for `type` within 2^-21, and 0 where it is below 2^-119), outputs as in
 * lq_norm_add with rows of heads * dim channels.
 *   o : [tokens][heads][dim] of `o_type` - binary32 from lq_decode_step and lq_scan_step, bf16 from lq_scan_prompt; strided rows
 *   z : [tokens][heads][dim] of `type`, strided rows      w : fp32 [dim] or null (1; LQ_NORM_RMS only)
 * No output may overlap an input or another output.
 */
typedef struct {
  int tokens, heads;
  int dim;     /* channels of a head: 64, 128 or 256 */
  int norm;
  int silu;
  int o_type;  /* lq_type of o          */
  int type;    /* lq_type of z and out  */
  float eps;
} lq_gated;
lq_status lq_norm_gate(const lq_gated *shape, const lq_norm_io *io, lq_stream stream);

/*
 * lq_product: rows of e4m3 codes times e4m3 weights, whose scales are of blocks of 128 output by 128 input channels:
 *     out[t][n] = sum_b x_scale[b][t] w_scale[n/128][b] sum_{k in block b} x[t][k] w[n][k]
 * The sum over a block is the tensor cores' (binary32 accumulator; off by 37 * 2^-23 of the sum over magnitudes at most, by one where the products are of
 * one size), the sum over blocks binary32; rounded once to `type`.
 *   x   : e4m3 [rows][in], strided rows, 16-byte aligned, stride a multiple of 16      x_scale : fp32 [ceil(in/128)][x_scale_stride]
 *   w   : e4m3 [out][in], dense, 16-byte aligned                                       w_scale : fp32 [ceil(out/128)][ceil(in/128)]
 *   out : [rows][out] of `type`, strided rows
 * `in` is a multiple of 16; in and out are at most 2^20, in * out and rows * x_stride below 2^40 (LQ_ERR_UNSUPPORTED beyond).
 * lq_product_groups: the rows of group g, group_start[g] to group_start[g+1] - 1 (int32 [groups + 1] in device memory, not decreasing), take
 * weight g: w [groups][out][in], w_scale [groups][ceil(out/128)][ceil(in/128)].  Groups may be empty; rows in front of group_start[0] and from
 * group_start[groups] on belong to nobody: they are not written, and what they hold does not matter.  At most LQ_MOST_GROUPS groups.
 * out must not overlap an input, group_start among them.  The order of all sums depends on the shapes and on group_start alone: the same call gives the same bits again.
 */
#define LQ_MOST_GROUPS 1024
typedef struct {
  int rows;
  int in, out;  /* channels                  */
  int groups;   /* lq_product: 1             */
  int type;     /* lq_type of out            */
} lq_linear;
typedef struct {
  const uint8_t *x;
  int64_t x_stride;
  const float *x_scale;
  int64_t x_scale_stride;
  const uint8_t *w;
  const float *w_scale;
  void *out;
  int64_t out_stride;
  const int32_t *group_start;   /* lq_product: not looked at */
} lq_product_io;
lq_status lq_product(const lq_linear *shape, const lq_product_io *io, lq_stream stream);
lq_status lq_product_groups(const lq_linear *shape, const lq_product_io *io, lq_stream stream);

/*
 * Device-side error flags of the current device (0 = none), written to *flags (a host pointer).  Waits inside
 * the kernels are bounded; bit 0 is set when a warp gave up waiting for its asynchronous copies (lq_scan_prompt, lq_product: or products), bit 1 when
 * one of these two did not find its shared or tensor memory where it counts on it (it then did nothing).  After
 * that, neither the outputs of that launch NOR THE STATE it worked on are valid (records may be missing or
 * half written): restore the state from a checkpoint.  Bit 3 belongs to lq_selftest_bounded_wait; the
 * others are not used.
 * The flags stay set until lq_clear_device_flags is called.  Both calls synchronise the device.
 */
lq_status lq_check_device(int *flags);
lq_status lq_clear_device_flags(void);

/*
 * Self test of the give-up path of the bounded waits (no passage of the paper): launches one warp that
 * waits, with a limit of 64 polls, on a barrier nothing completes.  The wait returns "gave up", the warp sets
 * bit 3 of the error flags and exits; the context stays usable.  Read the flag with lq_check_device and clear
 * it with lq_clear_device_flags.
 */
lq_status lq_selftest_bounded_wait(lq_stream stream);

/* LQ_STATIC_STAGE_BYTES as the loaded library was built with (for bindings that cannot read the macro). */
uint64_t lq_static_stage_bytes(void);

/* Kernels one lq_decode_step call launches (used to report launch counts; both 0 for an invalid shape):
 * lq_decode_launches: for `shape` on a state without scratch words, which is the most it launches;
 * lq_step_launches: on `state` as it is, which may be one where that is two. */
int lq_decode_launches(const lq_shape *shape);
int lq_step_launches(const lq_shape *shape, const lq_state *state);

const char *lq_status_string(lq_status status);
int lq_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LQ_H_ */
