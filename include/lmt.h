/* lmt.h -- operators at the two ends of a language model's training step, on one
 * MI355X (gfx950).  Part of libbca.so.
 *
 * bca.h takes gradients; these make the ones of the largest tensor a BERT-shaped
 * model has, the table of word pieces that is both the input's embedding and the
 * output's projection:
 *   lmt_embed           rows of the table for the tokens, scaled
 *   lmt_embed_grad      the table's gradient from the rows' gradients, tokens sorted
 *   lmt_quantize        a matrix (and its transpose) in 8-bit floating point with a
 *                       power of two for every 128 elements
 *   lmt_matmul          products of two such matrices: logits, gradients of inputs
 *                       and of weights
 *   lmt_cross_entropy   the loss of every row of logits and its gradient
 *
 * Conventions
 *   - 0 on success, negative LMT_ERR_* otherwise (nothing enqueued);
 *     lmt_last_error() has a message.  No call allocates, keeps state, synchronises
 *     or looks at DEVICE memory from the host: calls only enqueue kernels on `stream`
 *     (a hipStream_t as void*; NULL is the default stream) of the device that is
 *     current, where all their memory must lie, and can be captured in a HIP graph.
 *   - Matrices are row-major; a row stride (`ld`) is in elements and at least the row's
 *     length.  Floating-point matrices need only be aligned to their element size; the
 *     8-bit ones start on 16 bytes and have the fixed strides below.
 *   - Outputs may not overlap inputs or each other except where it is said.
 *   - Sums are in fp32 (but see lmt_matmul on 16-bit results) in an order that depends on the sizes, and for lmt_embed_grad
 *     the tokens, alone: the same call gives the same bits.
 *   - `status` (DEVICE int32, or NULL) has LMT_STATUS_* bits ORed in; the caller clears it,
 *     so that one word can watch many calls.
 */
#ifndef LMT_H_
#define LMT_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* element types; the first three as BCA_GRAD_* */
#define LMT_F32 0
#define LMT_F16 1
#define LMT_BF16 2
#define LMT_E4M3 3 /* 8 bits: 4 exponent, 3 mantissa, largest value 448, no infinities  */
#define LMT_E5M2 4 /* 8 bits: 5 exponent, 2 mantissa, largest value 57344               */
#define LMT_I32 5
#define LMT_I64 6

#define LMT_ERR_NULL (-1)      /* a required pointer is NULL                                     */
#define LMT_ERR_ARG (-2)       /* unknown type or flag, a stride below the row's length, no classes, scale not finite */
#define LMT_ERR_LIMIT (-3)     /* sizes beyond LMT_MAX_*                                         */
#define LMT_ERR_HIP (-4)       /* a HIP runtime call failed                                      */
#define LMT_ERR_ALIGN (-5)     /* a pointer is not aligned as it must be                         */
#define LMT_ERR_WORKSPACE (-6) /* the workspace is smaller than the call needs                   */

#define LMT_STATUS_BAD_TOKEN 1  /* a token outside [0, vocab): looked up as zeros, no gradient    */
#define LMT_STATUS_BAD_TARGET 2 /* a target outside [0, classes) that is not the ignored one: the row counts as ignored */

#define LMT_ACCUMULATE 1u  /* add to what the output holds                                           */
#define LMT_TILE_SCALES 2u /* lmt_quantize: one scale for a square of 128 x 128 instead of 128 x 1     */
#define LMT_FP32_SUMS 4u   /* lmt_matmul: a 16-bit c from sums as exact as an fp32 one's                */

#define LMT_MAX_ROWS 0x7fffff00u  /* tokens, vocabulary, rows, classes, m, n                     */
#define LMT_MAX_WIDTH 0x7fffffu   /* row length of tables and of 8-bit matrices, k                 */

/* out[t][j] = scale * table[token[t]][j] for t < n_tokens, j < width, rounded once to out's type.
 * table: [vocab][table_ld] of LMT_F32, _F16 or _BF16; tokens: [n_tokens] of LMT_I32 or LMT_I64;
 * out: [n_tokens][out_ld].  A token outside [0, vocab) gives a row of zeros and LMT_STATUS_BAD_TOKEN. */
int lmt_embed(const void* table /*DEVICE*/, int table_dtype, uint64_t vocab, uint64_t width, uint64_t table_ld,
              const void* tokens /*DEVICE*/, int token_dtype, uint64_t n_tokens, double scale, void* out /*DEVICE*/,
              int out_dtype, uint64_t out_ld, int32_t* status, void* stream);

/* Gradient of lmt_embed with respect to the table:
 *   grad[v][j] = (old grad[v][j], with LMT_ACCUMULATE) + scale * sum over t with token[t] == v of grad_out[t][j]
 * Without LMT_ACCUMULATE every row of grad is written, zeros where the token does not occur; with it only the rows that
 * occur are touched.  The tokens are sorted, equal ones kept in their order, so a row's sum never depends on timing.
 * `skip_token` has no gradient (the padding; any value outside [0, vocab) for none); nor has a token outside
 * [0, vocab), which is reported unless it is `skip_token`.  workspace: DEVICE, 16-byte aligned, at least
 * lmt_embed_grad_workspace bytes, contents of no concern; not shared by calls that overlap in time. */
uint64_t lmt_embed_grad_workspace(uint64_t n_tokens, uint64_t vocab, uint64_t width);
int lmt_embed_grad(const void* grad_out /*DEVICE*/, int grad_out_dtype, uint64_t grad_out_ld,
                   const void* tokens /*DEVICE*/, int token_dtype, uint64_t n_tokens, double scale, int64_t skip_token,
                   void* grad /*DEVICE*/, int grad_dtype, uint64_t vocab, uint64_t width, uint64_t grad_ld,
                   uint32_t flags, int32_t* status, void* workspace /*DEVICE*/, uint64_t workspace_bytes, void* stream);

/* The 8-bit form of a matrix of `rows` rows of `cols` elements.  Every row is cut into blocks of 128 elements;
 * lmt_fp8_row_bytes(cols) = 128 * ceil(cols / 128) bytes hold a row, zeros behind its end, and
 * lmt_scale_row_bytes(cols) = 4 * ceil(cols / 512) bytes its blocks' scales: byte e stands for 2^(e - 127),
 * 127 behind the last block.  Element j of row i is  q[i][j] * 2^(scales[i][j / 128] - 127). */
uint64_t lmt_fp8_row_bytes(uint64_t cols);
uint64_t lmt_scale_row_bytes(uint64_t cols);

/* x (fp32, fp16 or bf16, [rows][ld]) in 8 bits: q and scales, and / or its transpose, qt and scales_t (a matrix of `cols`
 * rows of `rows` elements, with blocks along its own rows).  Either pair may be NULL.  A block's scale is the smallest
 * power of two, at least 2^-126, that brings its largest finite magnitude to fp8's largest value or below (a block of
 * zeros: 2^-126); with LMT_TILE_SCALES the block is the square of 128 x 128 that the element lies in, so that the
 * transpose holds the same values.  Elements are rounded to the nearest value, ties to even; infinities and NaN become NaN
 * and take no part in the scale.  fp8: LMT_E4M3 or LMT_E5M2. */
int lmt_quantize(const void* x /*DEVICE*/, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int fp8, uint32_t flags,
                 void* q /*DEVICE*/, uint8_t* scales /*DEVICE*/, void* qt /*DEVICE*/, uint8_t* scales_t /*DEVICE*/,
                 void* stream);

/* c[i][j] = (old c[i][j], with LMT_ACCUMULATE) + sum over l < k of a[i][l] * b[j][l], for i < m, j < n, both operands in the
 * 8-bit form above with rows of k elements (each LMT_E4M3 or LMT_E5M2); c: fp32, fp16 or bf16, [m][ldc].  Products and sums are
 * made by the matrix cores and rounded once to c's type.  A 16-bit c takes the 8-bit instructions, which line up the products of
 * eight neighbours before they add them in fp32: of terms that are much smaller than their neighbours the last bits are lost, about 1.5e-5 of the
 * 2-norm of a result of normal numbers and up to 4e-5 where their magnitudes spread over e^2, at any k (a hundredth and a fortieth
 * of bf16's rounding, a fourteenth and a fifth of fp16's).  With LMT_FP32_SUMS it takes the bf16 instructions that an fp32 c always takes: exact products, sums
 * in fp32, at three to four fifths of the rate.  Those see an operand's elements as bf16 numbers: from 2^128 on infinite, below
 * 2^-130 exact to 2^-133 only.  a_scales and b_scales are 4-byte aligned and between 1 and 254.  workspace: as above, at
 * least lmt_matmul_workspace bytes; may be NULL where that is 0.
 * With x [T][H] and a weight w [V][H]: logits = x w^T are matmul(q(x), q(w)); the input's gradient dy w is
 * matmul(q(dy), qt(w)); the weight's dy^T x is matmul(qt(dy), qt(x)). */
uint64_t lmt_matmul_workspace(uint64_t m, uint64_t n, uint64_t k);
int lmt_matmul(const void* a /*DEVICE*/, int a_fp8, const uint8_t* a_scales /*DEVICE*/, const void* b /*DEVICE*/, int b_fp8,
               const uint8_t* b_scales /*DEVICE*/, uint64_t m, uint64_t n, uint64_t k, void* c /*DEVICE*/, int c_dtype,
               uint64_t ldc, uint32_t flags, void* workspace /*DEVICE*/, uint64_t workspace_bytes, void* stream);

/* Per row i of logits x (fp32, fp16 or bf16, [rows][ld]) with target t and weight w (weights[i], or 1 where weights is
 * NULL):
 *   lse[i] = log(sum over j of exp(x[j]));  loss[i] = w * (lse[i] - x[t]);  grad[i][j] = w * (exp(x[j] - lse[i]) - [j == t])
 * loss, lse (DEVICE [rows], fp32) and grad (DEVICE, the logits' type, [rows][grad_ld]; may be the logits themselves, with
 * their ld) may each be NULL.  A row whose target is `ignore` has loss 0 and a gradient of zeros, whatever its logits.
 * Logits of -Inf are classes that cannot occur; a row of nothing else has lse -Inf, loss +Inf and a gradient of
 * zeros.  +Inf and NaN make the row's results NaN. */
int lmt_cross_entropy(const void* logits /*DEVICE*/, int dtype, uint64_t rows, uint64_t classes, uint64_t ld,
                      const void* targets /*DEVICE*/, int target_dtype, int64_t ignore,
                      const float* weights /*DEVICE or NULL*/, float* loss, float* lse, void* grad, uint64_t grad_ld,
                      int32_t* status, void* stream);

/* Message of the calling thread's last error; valid until its next call. */
const char* lmt_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* LMT_H_ */
