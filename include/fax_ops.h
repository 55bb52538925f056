/*
 * fax_ops.h -- operator-level entry points of the same library: the single
 * kernels the block and LM step are made of, exposed so that each can be
 * checked against the oracle and timed against its roofline on its own.
 * All conventions of fax.h hold (device pointers, caller-owned buffers,
 * asynchronous on the context's stream, fax_status results).  "T" is bf16 for
 * FAX_PREC_BF16 and float for FAX_PREC_FP32_VALIDATE.
 */
#ifndef FAX_OPS_H_
#define FAX_OPS_H_

#include "fax.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Epilogues of the GEMM (the fused tails the block's linear layers need). */
enum {
  FAX_EPI_NONE = 0,        /* C = alpha * A B                                     */
  FAX_EPI_BIAS = 1,        /* C = alpha * A B + bias[n]                           */
  FAX_EPI_BIAS_GELU = 2,   /* C = alpha * A B + bias (stored), aux = GELU_tanh(C) */
  FAX_EPI_BIAS_RESID = 3,  /* C = alpha * A B + bias + resid                      */
  FAX_EPI_DGELU = 4        /* C = (alpha * A B) * GELU_tanh'(aux)                 */
};

/* C[M,N] = op(A) op(B) with float accumulation -- the QKV, attention-output,
 * MLP and output-head contractions of the step and their backward forms
 * (Sec. 3.2: the large matrix multiplications of the transformer).
 * A is [M,K] row-major (a_mn_major = 0) or [K,M] row-major (a_mn_major = 1);
 * B is [N,K] row-major (b_mn_major = 0) or [K,N] row-major (b_mn_major = 1);
 * lda / ldb / ldc / ldr / ldaux are row strides in elements.  C is T, or
 * float when c_f32 != 0; accumulate != 0 adds into a float C.  bias [N],
 * resid [M,N] and aux [M,N] are T.  In FAX_PREC_BF16 the problem runs on the
 * tensor-core kernels (M a multiple of 128, N and K of 64, 16-byte aligned rows)
 * and any other shape is refused with FAX_ERR_UNSUPPORTED_SHAPE: it never lands
 * on the far slower float-FMA kernel unasked.  force_simt != 0 selects that
 * kernel, for any shape and in either precision (FAX_PREC_FP32_VALIDATE always
 * uses it). */
typedef struct {
  int32_t M, N, K;
  const void* A; int64_t lda; int32_t a_mn_major;
  const void* B; int64_t ldb; int32_t b_mn_major;
  void* C; int64_t ldc; int32_t c_f32; int32_t accumulate;
  int32_t epilogue;
  const void* bias;
  const void* resid; int64_t ldr;
  void* aux; int64_t ldaux;
  float alpha;
  int32_t force_simt;
} fax_gemm_desc;

fax_status fax_op_gemm(fax_ctx* ctx, int32_t prec, const fax_gemm_desc* desc);

/* Row-wise LayerNorm over d (biased variance, eps inside the square root):
 * out = gamma * (x - mu) * rstd + beta; mu, rstd [rows] float are saved. */
fax_status fax_op_layernorm_forward(fax_ctx* ctx, int32_t prec, int32_t rows, int32_t d, const void* x,
                                    const void* gamma, const void* beta, float eps, void* out,
                                    float* mu, float* rstd);

/* Reverse of the above: dx = (add ? add : 0) + dLN(da); dgamma, dbeta [d]
 * float are overwritten.  scratch: fax_op_layernorm_backward_scratch_bytes. */
fax_status fax_op_layernorm_backward_scratch_bytes(int32_t rows, int32_t d, size_t* bytes);
fax_status fax_op_layernorm_backward(fax_ctx* ctx, int32_t prec, int32_t rows, int32_t d, const void* da,
                                     const void* x, const float* mu, const float* rstd, const void* gamma,
                                     const void* add, void* dx, float* dgamma, float* dbeta,
                                     void* scratch, size_t scratch_bytes);

/* LayerNorm backward without caller scratch and without any allocation.  (The
 * paper has no counterpart of this call; it exists for deployment reasons.)
 * Some hosts of this library cannot give it scratch memory or let it call
 * cudaMalloc: a serving or training process whose own pool already owns all
 * device memory, a plug-in that runs under a fixed memory budget, or a
 * latency-critical loop that cannot afford the device-wide synchronisation an
 * allocation implies.  For them the column-sum partials of dgamma / dbeta live
 * in a fixed array inside the library image: FAX_LN_STATIC_SCRATCH_FLOATS
 * floats (8 MiB), resident on every GPU that loads the library until the
 * process exits.  The call computes exactly what fax_op_layernorm_backward
 * computes (same kernels) and calls no cudaMalloc, cudaFree or allocating
 * library routine.
 *  - Limit: d <= FAX_LN_STATIC_MAX_D (4096) at any row count (the array holds
 *    the partial sums of up to 256 row slabs of that width); a wider row makes
 *    the call do nothing and return FAX_ERR_WORKSPACE_TOO_SMALL.
 *  - The first call on each device looks the array's device address up (one
 *    cudaGetSymbolAddress with that device current).  Make that first call
 *    before starting any stream capture on the device.
 *  - All calls on a device share the one array, and it keeps whatever the last
 *    call left.  Nothing in it needs clearing (every slot is written before it
 *    is read), but two calls whose kernels overlap on the GPU (different
 *    streams or contexts) race on it: serialise them. */
#define FAX_LN_STATIC_MAX_D 4096
#define FAX_LN_STATIC_SCRATCH_FLOATS (2 * 256 * FAX_LN_STATIC_MAX_D)
fax_status fax_op_layernorm_backward_static(fax_ctx* ctx, int32_t prec, int32_t rows, int32_t d, const void* da,
                                            const void* x, const float* mu, const float* rstd,
                                            const void* gamma, const void* add, void* dx, float* dgamma,
                                            float* dbeta);

/* Causal multi-head attention (Sec. 3.2: multi-headed attention blocks) on a
 * fused qkv [batch*seq, 3*n_heads*head_dim] T buffer (layout in fax.h):
 * o [batch*seq, n_heads*head_dim] T, lse [batch, n_heads, seq] float
 * (natural-log sum of exponentials of the scaled, masked scores). */
fax_status fax_op_attention_forward(fax_ctx* ctx, int32_t prec, int32_t batch, int32_t seq, int32_t n_heads,
                                    int32_t head_dim, const void* qkv, void* o, float* lse);

/* Reverse: given d_o [batch*seq, d] T writes dqkv [batch*seq, 3d] T. */
fax_status fax_op_attention_backward_scratch_bytes(int32_t prec, int32_t batch, int32_t seq,
                                                   int32_t n_heads, int32_t head_dim, size_t* bytes);
fax_status fax_op_attention_backward(fax_ctx* ctx, int32_t prec, int32_t batch, int32_t seq,
                                     int32_t n_heads, int32_t head_dim, const void* qkv, const void* o,
                                     const float* lse, const void* d_o, void* dqkv, void* scratch,
                                     size_t scratch_bytes);

/* Token table lookup: out[i, :] = scale * table[ids[i], :], rounded once to T.
 * ids: n_tokens int32; an id outside [0, vocab) (padding) gives a row of zeros.
 * table [vocab, d] T, out [n_tokens, d] T.  n_tokens = 0 does nothing; n_tokens and d <= 2^30. */
fax_status fax_op_embedding_forward(fax_ctx* ctx, int32_t prec, int32_t n_tokens, int32_t vocab, int32_t d,
                                    const int32_t* ids, const void* table, float scale, void* out);

/* Its reverse: dtable[v, :] = scale * sum over the tokens i with ids[i] = v of
 * dout[i, :]  (accumulate != 0: added to what dtable holds, e.g. the output
 * head's gradient of a tied table).  dout [n_tokens, d] T; dtable [vocab, d]
 * float: overwritten in full, or with accumulate != 0 changed only in rows
 * that a token touches.  Tokens with an id outside [0, vocab) add nothing.  Each
 * row is summed over its tokens in float32 in a fixed order (long batches are
 * sorted by id first, short ones are not): the same inputs give the same bits (an accumulated row gets its sum in
 * one addition per element, in memory, where subnormal numbers count as 0).  Concurrent calls, and graphs that may be replayed at
 * the same time, need scratch of their own.  n_tokens and d <= 2^30; scratch 256-byte aligned.
 * Scratch of the longest batch serves every shorter one: the bytes never shrink with n_tokens, vocab or d. */
fax_status fax_op_embedding_backward_scratch_bytes(int32_t n_tokens, int32_t vocab, int32_t d, size_t* bytes);
fax_status fax_op_embedding_backward(fax_ctx* ctx, int32_t prec, int32_t n_tokens, int32_t vocab, int32_t d,
                                     const int32_t* ids, const void* dout, float scale, int32_t accumulate,
                                     float* dtable, void* scratch, size_t scratch_bytes);

/* ---- matrices in 8-bit floating point, and their products ----
 * A matrix is held as one byte an element (FAX_FP8_E4M3: largest value 448;
 * FAX_FP8_E5M2: 57344; both with NaN 0x7f) and a float32 scale for each 1 x 128
 * (tile 1) or 128 x 128 (tile 128) block of it: element = scale * value.  Blocks
 * begin at row 0 and column 0; those at the edges are cut off.  The scales of a
 * matrix [R, C] are stored with the block of columns first:
 * scale[(c / 128) * ld + r] (tile 1, ld >= R) or
 * scale[(c / 128) * ld + r / 128] (tile 128, ld >= ceil(R / 128)). */
enum { FAX_FP8_E4M3 = 0, FAX_FP8_E5M2 = 1 };
#define FAX_FP8_BLOCK 128

/* x [rows, cols] T with row pitch ldx -> any of
 *   q  [rows, cols] with pitch ldq and its scales s, pitch lds     (NULL: not wanted)
 *   qt [cols, rows], x transposed, pitch ldqt, its scales st, pitch ldst
 *                    (blocks along x's columns: tokens, for a weight gradient)
 * from one reading of x.  A block's scale is the smallest power of two, at least
 * 2^-126, that brings its largest finite magnitude to the format's largest value
 * at most (1 for a block without any above 0); values are x / scale (exact)
 * rounded to nearest even; elements that are not finite become NaN.  ldq and
 * ldqt are multiples of 16, q and qt 16-byte aligned; bytes between cols and ldq
 * (rows and ldqt) are left as they were. */
typedef struct {
  int32_t rows, cols;
  const void* x; int64_t ldx;
  int32_t format, tile;
  void* q; int64_t ldq; float* s; int64_t lds;
  void* qt; int64_t ldqt; float* st; int64_t ldst;
} fax_fp8_quantize_desc;
fax_status fax_op_fp8_quantize(fax_ctx* ctx, int32_t prec, const fax_fp8_quantize_desc* desc);

/* C[M, N] = A B^T of two such matrices, A [M, K] with tile 1 and B [N, K] with
 * b_tile 1 or 128, both row-major with pitches lda, ldb (multiples of 16;
 * 16-byte aligned bases), formats chosen for each:
 *   C[m, n] = sum over blocks b of 128 k of sa[b, m] sb[b, n] sum_{k in b} A[m, k] B[n, k]
 * in float32 on the tensor cores, plus bias[n] (bf16; NULL: none), rounded once
 * to bf16, or kept as float (c_f32 != 0), or added to a float C (accumulate != 0).
 * The forward product takes activations and transposed weights (tile 128),
 * the input gradient output gradients and weights as stored, the weight gradient
 * both factors transposed with tile 1.  Any M, N, K from 1 on.  What is added to
 * C is added in memory, where subnormal numbers count as 0 (on either side and in
 * the sum).  The scales are powers of
 * two from 2^-126 to 2^127, as fax_op_fp8_quantize gives them (of any other
 * float the exponent alone counts; infinities and NaN make NaN).  ldc >= N in elements; C aligned to its
 * elements (16-byte aligned rows are stored faster).  C may not overlap A or B. */
typedef struct {
  int32_t M, N, K;
  const void* A; int64_t lda; int32_t a_format; const float* a_scale; int64_t a_scale_ld;
  const void* B; int64_t ldb; int32_t b_format; const float* b_scale; int64_t b_scale_ld; int32_t b_tile;
  void* C; int64_t ldc; int32_t c_f32; int32_t accumulate;
  const void* bias;
} fax_fp8_gemm_desc;
fax_status fax_op_fp8_gemm(fax_ctx* ctx, const fax_fp8_gemm_desc* desc);

/* The tile that fax_op_fp8_gemm takes for a product of these sizes under the context's settings (host pointers): how
 * many SMs share one (1, or 2: a pair, unless fax_set_gemm_two_cta is off), its columns (64 to 256; 128 rows an SM), and
 * the slices of K that a cluster of SMs joins (1: none).  For inspection and tests; nothing is launched. */
fax_status fax_op_fp8_gemm_tile(const fax_ctx* ctx, int32_t M, int32_t N, int32_t K, int32_t c_f32,
                                int32_t* sms, int32_t* columns, int32_t* slices);

/* ---- positions by rotation ----
 * The first rot_dim elements of each head are rot_dim / 2 pairs, (i, i + rot_dim / 2) with FAX_ROTARY_HALVES or
 * (2i, 2i + 1) with FAX_ROTARY_PAIRS; pair i of a token at position p is turned by the angle p * frequency[i]:
 *   y_a = amplitude * (cos * x_a - sin * x_b),   y_b = amplitude * (cos * x_b + sin * x_a)
 * (backward != 0: sin negated, which is the gradient: dx from dy).  The elements behind rot_dim are copied, or stay
 * where y is x.  x [rows, heads * head_dim] T, pitch ldx: `heads` heads one after another, e.g. q and k (2 * n_heads) of a fused
 * qkv buffer; y likewise with pitch ldy, x itself (ldy = ldx) or memory that holds none of x's elements.  A token's position
 * is positions[row] (int32, device), or without positions first + row % seq (seq = 0: first + row).  frequencies: device,
 * rot_dim / 2 words from fax_rotary_frequencies.  The angle is exact modulo a turn at any position (whole numbers
 * modulo 2^64); y is rounded once to T.  rows = 0 does nothing; rot_dim is even,
 * head_dim <= FAX_ROTARY_MAX_DIM and, where y is not x, even too; rows <= 2^30, heads * head_dim <= 2^24. */
enum { FAX_ROTARY_HALVES = 0, FAX_ROTARY_PAIRS = 1 };
#define FAX_ROTARY_MAX_DIM 1024
typedef struct {
  int32_t rows, heads, head_dim, rot_dim, layout;
  const void* x; int64_t ldx;
  void* y; int64_t ldy;
  const int32_t* positions; int32_t first, seq;
  const uint64_t* frequencies;
  float amplitude;
  int32_t backward;
} fax_rotary_desc;
fax_status fax_op_rotary(fax_ctx* ctx, int32_t prec, const fax_rotary_desc* desc);

/* frequency[i] = base^(-2 i / rot_dim) radians a position, as turns in units of 2^-64 (host, rot_dim / 2 words).
 * For contexts `factor` times longer than trained: original_seq = 0 divides every frequency by factor; original_seq > 0
 * keeps pairs that make high_turns or more turns in original_seq tokens, divides those of low_turns or fewer by factor
 * and goes linearly in the turns between.  base >= 1, factor >= 1 (1: no scaling, the rest is not looked at), low_turns < high_turns. */
fax_status fax_rotary_frequencies(int32_t rot_dim, double base, double factor, int32_t original_seq, double low_turns,
                                  double high_turns, uint64_t* frequencies_host);

/* ---- dropout ----
 * y = resid + (kept ? x / (1 - p) : 0), rounded once to T (resid NULL: without it; a dropped element's x is not
 * looked at).  An element is dropped where its 16 random bits are below round(65536 p); 1 - p is taken as
 * 1 - round(65536 p) / 65536, so that the mean is x.  The bits are those of Philox4x32-10 (Salmon, Moraes, Dror,
 * Shaw 2011) under the key `seed` for the counter (column / 8, row, offset), two 32-bit words of offset, low ones
 * first: elements 2 w and 2 w + 1 of the eight columns have the low and the high half of word w.  Nothing is stored: the gradient is the
 * same call on dy without resid.  Where offset_device is not NULL the 64-bit word there is added to offset when the kernel
 * runs, so that a captured graph draws anew at each replay.  x, resid, y [rows, cols] T with pitches; y may be x
 * or resid (same pitch), otherwise it holds none of their elements.  0 <= p <= 1 (1: nothing is kept); rows = 0 does nothing. */
typedef struct {
  int32_t rows, cols;
  const void* x; int64_t ldx;
  const void* resid; int64_t ldr;
  void* y; int64_t ldy;
  float p;
  uint64_t seed, offset;
  const uint64_t* offset_device;
} fax_dropout_desc;
fax_status fax_op_dropout(fax_ctx* ctx, int32_t prec, const fax_dropout_desc* desc);

/* ---- gated linear recurrence ----
 * For each channel c of d and the tokens t of a sequence, in float32:
 *   a_t = 1 / (1 + exp(-f_t))      h_t = a_t h_{t-1} + b_t      y_t = h_t, or with g: h_t g_t / (1 + exp(-g_t))
 * with b_t = x_t (FAX_RECURRENCE_PLAIN) or (1 - a_t) x_t (FAX_RECURRENCE_COMPLEMENT).  With bf16
 * inputs the exponentials and reciprocals are the hardware's approximations: a sigmoid of f, and 1 less it, is off by
 * (2^-21 + 2^-23 |f|) of itself and 2^-126 at most, which h_last, states and dh0 inherit.  h starts at h0 [n_seq, d] float
 * (NULL: zeros) and ends in h_last [n_seq, d] float (NULL: not wanted; may be h0), so that a sequence can be continued, a
 * token at a time too.  f, x, g (NULL: none), y are [rows, d] T with pitches (columns of one fused projection, e.g.).
 * Sequences are `seq` rows each (rows = n_seq * seq), or with offsets (device, [n_seq + 1] int32, not falling, within 0 to rows) sequence s is
 * rows offsets[s] to offsets[s + 1] - 1, with seq the longest one's length (a choice of kernel goes by it, and with it the
 * order of roundings); rows outside stay as they were.  Offsets outside [0, rows] are taken as the nearest end, a falling one
 * as an empty sequence.  Where a sequence behind a falling offset begins before the end of an earlier one, nothing but the arrays is
 * touched, but y of rows that both have, and whatever the backward pass makes of the call, have no meaning (each writes, in no order).
 * states: NULL, or for the backward pass fax_op_recurrence_states_floats floats, which receive h before every 16th token.
 * y holds no element of f, x or g.  The same call on the same device gives the same bits.  rows = 0 still writes h_last.  rows <= 2^30,
 * d <= 2^24, n_seq * ceil(d / 64) <= 2^27 - 1. */
enum { FAX_RECURRENCE_PLAIN = 0, FAX_RECURRENCE_COMPLEMENT = 1 };
#define FAX_RECURRENCE_BLOCK 16
typedef struct {
  int32_t rows, d, n_seq, seq;
  const int32_t* offsets;
  int32_t input;
  const void* f; int64_t ldf;
  const void* x; int64_t ldx;
  const void* g; int64_t ldg;
  const float* h0;
  void* y; int64_t ldy;
  float* h_last;
  float* states;
} fax_recurrence_desc;
fax_status fax_op_recurrence_states_floats(int32_t rows, int32_t n_seq, int32_t d, size_t* floats);
fax_status fax_op_recurrence_forward(fax_ctx* ctx, int32_t prec, const fax_recurrence_desc* desc);

/* Its reverse: from dy [rows, d] T and dh_last [n_seq, d] float (NULL: zeros), with the forward call's inputs, states and
 * sequences: df, dx, dg (wanted with g) [rows, d] T, and dh0 [n_seq, d] float (NULL: not wanted; may be dh_last).
 *   dh_t = dy_t (g_t / (1 + exp(-g_t)) or 1) + a_{t+1} dh_{t+1}      dh0 = a_1 dh_1
 * The gradients' memory holds no element of the inputs, except that each may be the input it belongs to (df f, dx x,
 * dg g; same pitch). */
typedef struct {
  int32_t rows, d, n_seq, seq;
  const int32_t* offsets;
  int32_t input;
  const void* f; int64_t ldf;
  const void* x; int64_t ldx;
  const void* g; int64_t ldg;
  const float* h0;
  const float* states;
  const void* dy; int64_t lddy;
  const float* dh_last;
  void* df; int64_t lddf;
  void* dx; int64_t lddx;
  void* dg; int64_t lddg;
  float* dh0;
} fax_recurrence_backward_desc;
fax_status fax_op_recurrence_backward(fax_ctx* ctx, int32_t prec, const fax_recurrence_backward_desc* desc);

/* ---- a feed-forward layer of experts: tokens to their experts and back ----
 * ids [n_tokens, top_k] int32: the experts a token chose; choices outside [0, n_experts) (padding) go nowhere.
 * Each choice gets a slot, a row of a buffer in which every expert's tokens are together, in the order of
 * (token, choice).  capacity > 0: expert e has the slots from e * capacity on, choices beyond its capacity go
 * nowhere (the latest ones).  capacity = 0: an expert has as many slots as choices, rounded up to a multiple of
 * `align` (e.g. 128 for fax_op_gemm).  Written: slot_of [n_tokens, top_k] (-1: nowhere), source [slots] (token * top_k +
 * choice, -1: empty), offsets [n_experts + 1] (first slot of each expert), counts [n_experts] (choices
 * made, kept or not), all int32.  slots is the length of source and the rows of the buffer, at least fax_op_expert_slots'.
 * n_experts <= FAX_EXPERT_MAX; n_tokens = 0 gives an empty plan. */
#define FAX_EXPERT_MAX 1024
typedef struct {
  int32_t n_tokens, top_k, n_experts, capacity, align, slots;
  const int32_t* ids;
  int32_t* slot_of;
  int32_t* source;
  int32_t* offsets;
  int32_t* counts;
} fax_expert_sort_desc;
fax_status fax_op_expert_slots(int32_t n_tokens, int32_t top_k, int32_t n_experts, int32_t capacity, int32_t align,
                               int32_t* slots_host);
fax_status fax_op_expert_sort(fax_ctx* ctx, const fax_expert_sort_desc* desc);

/* out[slot] = x[token] for every choice that has a slot, zeros in empty slots: all `slots` rows are written.
 * x [n_tokens, d] T, out [slots, d] T, with pitches.  Its reverse is fax_op_expert_combine without weights.
 * In all three calls a slot_of outside [0, slots) counts as -1. */
typedef struct {
  int32_t n_tokens, top_k, d, slots;
  const int32_t* slot_of;
  const int32_t* source;
  const void* x; int64_t ldx;
  void* out; int64_t ldo;
} fax_expert_dispatch_desc;
fax_status fax_op_expert_dispatch(fax_ctx* ctx, int32_t prec, const fax_expert_dispatch_desc* desc);

/* y[token] = resid[token] (NULL: 0) + sum over its choices j, in their order, of weights[token, j] (NULL: 1) *
 * z[slot_of[token, j]], in float32, rounded once to T.  weights [n_tokens, top_k] float; z [slots, d], resid and
 * y [n_tokens, d] T, with pitches; y may be resid (same pitch). */
typedef struct {
  int32_t n_tokens, top_k, d, slots;
  const int32_t* slot_of;
  const float* weights;
  const void* z; int64_t ldz;
  const void* resid; int64_t ldr;
  void* y; int64_t ldy;
} fax_expert_combine_desc;
fax_status fax_op_expert_combine(fax_ctx* ctx, int32_t prec, const fax_expert_combine_desc* desc);

/* Its reverse (resid's gradient is dy): dz[slot] = weights[token, j] * dy[token], zeros in empty slots (all `slots`
 * rows are written); dw[token, j] = sum over d of z[slot] dy[token], 0 for a choice without a slot (NULL: not wanted;
 * z is not read then).  dz [slots, d] T, dw [n_tokens, top_k] float; dz may be z (same pitch). */
typedef struct {
  int32_t n_tokens, top_k, d, slots;
  const int32_t* slot_of;
  const int32_t* source;
  const float* weights;
  const void* z; int64_t ldz;
  const void* dy; int64_t lddy;
  void* dz; int64_t lddz;
  float* dw;
} fax_expert_combine_backward_desc;
fax_status fax_op_expert_combine_backward(fax_ctx* ctx, int32_t prec, const fax_expert_combine_backward_desc* desc);

#ifdef __cplusplus
}
#endif
#endif /* FAX_OPS_H_ */
