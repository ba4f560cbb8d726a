/* lmt.h -- operators at the two ends of a language model's training step and of the
 * attention between them, on one MI355X (gfx950).  Part of libbca.so.
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
 *   lmt_linear_cross_entropy  the same from the rows and the table, with the gradients of
 *                       both, the logits not kept
 * and these mix the rows of sequences of unlike lengths:
 *   lmt_rotary          queries and keys turned by their positions; its gradient
 *   lmt_attention       attention within each sequence of a packed or padded batch
 *   lmt_attention_grad  gradients of its queries, keys and values
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
#define LMT_ERR_LIMIT (-3)     /* sizes beyond LMT_MAX_*, or more than a launch can have         */
#define LMT_ERR_HIP (-4)       /* a HIP runtime call failed                                      */
#define LMT_ERR_ALIGN (-5)     /* a pointer is not aligned as it must be                         */
#define LMT_ERR_WORKSPACE (-6) /* the workspace is smaller than the call needs                   */

#define LMT_STATUS_BAD_TOKEN 1  /* a token outside [0, vocab): looked up as zeros, no gradient    */
#define LMT_STATUS_BAD_TARGET 2 /* a target outside [0, classes) that is not the ignored one: the row counts as ignored */
#define LMT_STATUS_BAD_SEQUENCE 4 /* starts that fall or leave the rows, or a length that reaches into the next sequence: cut to what is there */

#define LMT_ACCUMULATE 1u  /* add to what the output holds                                           */
#define LMT_TILE_SCALES 2u /* lmt_quantize: one scale for a square of 128 x 128 instead of 128 x 1     */
#define LMT_FP32_SUMS 4u   /* lmt_matmul: a 16-bit c from sums as exact as an fp32 one's                */
#define LMT_NEIGHBOURS 8u  /* lmt_rotary: pairs of neighbours instead of elements `pairs` apart        */
#define LMT_INVERSE 16u    /* lmt_rotary: turns back (the gradient)                                    */
#define LMT_CAUSAL 32u     /* attention: no position sees a later one, but for prefixes                */

#define LMT_MAX_HEAD 128u         /* elements of a head                                          */
#define LMT_MAX_HEADS 65535u
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

/* lmt_cross_entropy of the logits x table^T, which are not kept:
 *   l[i][j] = sum over m of x[i][m] table[j][m];  lse, loss as above;  g[i][j] = w (exp(l[i][j] - lse[i]) - [j == t])
 *   grad_x = g table;  grad_table = (old grad_table, with LMT_ACCUMULATE) + g^T x
 * x: [rows][x_ld], table: [classes][table_ld], both of `dtype`, LMT_F16 or LMT_BF16; rows, classes and width are up to LMT_MAX_WIDTH.  Logits, losses and
 * sums are in fp32; elements of g are rounded to `dtype` before they are multiplied (fp16: scaled by powers of two, for grad_x in front of the row's weight and for
 * grad_table with it, and never off by more than 2^-39 of the row's weight in the one and 2^-38 of the largest in the other beside a rounding); with up to 256 rows what that
 * leaves is multiplied too.  loss, lse (DEVICE [rows], fp32), grad_x (of `dtype`, [rows][grad_x_ld]) and grad_table (of grad_table_dtype,
 * `dtype` or LMT_F32, [classes][grad_table_ld]) may each be NULL.  Ignored rows have no loss, a grad_x of zeros and no part in grad_table, whatever they
 * hold; their lse is that of any row.
 * Infinities and NaN in a row of x or in its weight are in that row's results and in grad_table; those in a row of the table are in everything.
 * What is kept instead of the logits is g, for at most 2^27 logits at a time (256 MB; in fp16 again without weights; with up to 256 rows again for what rounding leaves), beside
 * fp32 sums of grad_x, a copy of the counted rows of x, and copies of x and the table where their rows do not lie as the kernels read them (width no multiple of 64, or not on 16
 * bytes).  So the workspace does not grow with rows x classes (but for 8 bytes a row and 128 or 256 classes); below 2^27 logits it is no less than logits in 16 bits.
 * workspace: DEVICE, 16-byte aligned, contents of no concern; not shared by calls that overlap in time.  lmt_linear_cross_entropy_workspace bytes (with gradients != 0
 * if grad_x or grad_table is given) are enough for any call of these sizes; lmt_linear_cross_entropy_workspace_of is what one of `dtype` needs whose x and table start on 16 bytes
 * and have strides that are multiples of 8.  Without rows a grad_table that is not added to is refused. */
uint64_t lmt_linear_cross_entropy_workspace(uint64_t rows, uint64_t classes, uint64_t width, int gradients);
uint64_t lmt_linear_cross_entropy_workspace_of(int dtype, uint64_t rows, uint64_t classes, uint64_t width, int gradients);
int lmt_linear_cross_entropy(const void* x /*DEVICE*/, uint64_t x_ld, const void* table /*DEVICE*/, uint64_t table_ld, int dtype,
                             uint64_t rows, uint64_t classes, uint64_t width, const void* targets /*DEVICE*/, int target_dtype,
                             int64_t ignore, const float* weights /*DEVICE or NULL*/, float* loss, float* lse, void* grad_x,
                             uint64_t grad_x_ld, void* grad_table, int grad_table_dtype, uint64_t grad_table_ld, uint32_t flags,
                             int32_t* status, void* workspace /*DEVICE*/, uint64_t workspace_bytes, void* stream);

/* Rows (tokens) of heads: element j of head h of row i is at[i * row + h * head + j], strides in elements, so that the parts
 * of one projection's output, and heads in front of rows, are taken as they lie.  Inputs may repeat rows or heads (strides of
 * 0); elements of outputs may not coincide.  `at` is DEVICE and aligned to an element; nothing is written through that of an input. */
typedef struct lmt_heads {
  void* at;
  uint64_t row, head;
} lmt_heads;

/* The first 2 * pairs elements of every head (size elements, at most LMT_MAX_HEAD) in pairs (a, b), pair f being elements f and
 * f + pairs, or with LMT_NEIGHBOURS 2 f and 2 f + 1:
 *   a' = m (a cos z - b sin z),  b' = m (a sin z + b cos z),  z = positions[i] * frequencies[f], or - z with LMT_INVERSE
 * The rest of a head is copied.  The gradient of a call is the call with the same m and the other direction.  x, out: `dtype`
 * (LMT_F32, LMT_F16, LMT_BF16), rows x heads; out may be x itself.  positions: [rows] of LMT_I32 or LMT_I64; frequencies:
 * [pairs], fp32, radians.  The angle is made in 64 bits, so that far positions keep theirs. */
int lmt_rotary(const lmt_heads* x, int dtype, uint64_t rows, uint64_t heads, uint64_t size, const void* positions /*DEVICE*/,
               int position_dtype, const float* frequencies /*DEVICE*/, uint64_t pairs, double magnitude, uint32_t flags,
               const lmt_heads* out, void* stream);

/* What attention goes by.  Sequence s has the rows from starts[s] on, lengths[s] of them or (lengths NULL) those up to starts[s + 1];
 * starts rise from 0 or above to `rows` or below, a sequence ends before the next one begins, and both are read on the device. */
typedef struct lmt_attend {
  int32_t dtype;                          /* of all elements: LMT_F16 or LMT_BF16                                          */
  uint32_t flags;                         /* LMT_CAUSAL                                                                    */
  uint64_t rows, heads, kv_heads, size;   /* query heads h use key head h / (heads / kv_heads); size <= LMT_MAX_HEAD        */
  uint64_t sequences;
  const int32_t *starts /*DEVICE [sequences + 1]*/, *lengths /*DEVICE [sequences] or NULL*/;
  const int32_t* prefixes;                /* DEVICE [sequences] or NULL, with LMT_CAUSAL: all of a sequence sees its first prefixes[s] positions */
  const float* slopes;                    /* DEVICE [heads] or NULL                                                        */
  double scale, cap;                      /* cap: 0 for none;  1.5 times either, and scale / cap, are finite in fp32       */
  int32_t* status;                        /* DEVICE or NULL                                                                */
} lmt_attend;

/* For every row i and head h, over the rows j of i's sequence that it sees (all, or with LMT_CAUSAL j <= i and the prefix):
 *   s[j] = scale * (q[i] . k[j]), then cap * tanh(s / cap) if there is a cap, then - slopes[h] * |i - j|
 *   out[i] = sum over j of exp(s[j] - lse) v[j];  lse[h][i] = log(sum over j of exp(s[j]))
 * q, out: rows x heads; k, v: rows x kv_heads; lse: DEVICE [heads][rows], fp32, or NULL.  Rows of no sequence, and rows all of whose
 * scores are -Inf, get zeros and an lse of -Inf.  What a row does not see has no part in its results, whatever it holds (rows that
 * infinities or NaN reach are computed once more, one after the other: 0.2 to 0.4 ns for each row and each that it sees, a head, twice that for the gradients; one NaN that all of a sequence of
 * 8 192 rows and 16 heads sees, 0.2 s and 0.4 s instead of a millisecond).  Scores, weights' sums and outputs' sums are in fp32, the weights that multiply v
 * are rounded to `dtype`. */
int lmt_attention(const lmt_attend* a, const lmt_heads* q, const lmt_heads* k, const lmt_heads* v, const lmt_heads* out,
                  float* lse, void* stream);

/* Gradients of lmt_attention with respect to q, k and v from that of out.  out and lse are what lmt_attention left for the same `a`.
 *   d[j] = p[j] (grad_out[i] . v[j] - grad_out[i] . out[i]),  p[j] = exp(s[j] - lse),  times 1 - (s / cap)^2 behind a cap
 *   grad_q[i] = scale * sum over j of d[j] k[j];  grad_k[j] = scale * sum over i of d[j] q[i];  grad_v[j] = sum over i of p[j] grad_out[i]
 * A key head's gradients are sums over the query heads that use it.  Rows of no sequence get zeros.  p and d are rounded to `dtype`
 * before they are multiplied (fp16: d scaled by a power of two that follows the largest of its row, of q for grad_q and of k for grad_k).  workspace: DEVICE, 16-byte aligned, at least
 * lmt_attention_grad_workspace bytes, contents of no concern; not shared by calls that overlap in time. */
uint64_t lmt_attention_grad_workspace(uint64_t rows, uint64_t heads, uint64_t kv_heads, uint64_t size);
int lmt_attention_grad(const lmt_attend* a, const lmt_heads* grad_out, const lmt_heads* q, const lmt_heads* k, const lmt_heads* v,
                       const lmt_heads* out, const float* lse, const lmt_heads* grad_q, const lmt_heads* grad_k,
                       const lmt_heads* grad_v, void* workspace /*DEVICE*/, uint64_t workspace_bytes, void* stream);

/* Message of the calling thread's last error; valid until its next call. */
const char* lmt_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* LMT_H_ */
