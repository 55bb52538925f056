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

#ifdef __cplusplus
}
#endif
#endif /* FAX_OPS_H_ */
