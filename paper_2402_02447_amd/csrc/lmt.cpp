// Host side of lmt.h: argument checks and the C entry points.  Nothing here allocates or throws.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "lmt_internal.h"

namespace {

thread_local char g_error[256] = "";
__attribute__((format(printf, 2, 3))) int fail(int code, const char* format, ...) {
  va_list args;
  va_start(args, format);
  vsnprintf(g_error, sizeof g_error, format, args);
  va_end(args);
  return code;
}

bool is_float(int t) { return t == LMT_F32 || t == LMT_F16 || t == LMT_BF16; }
bool is_fp8(int t) { return t == LMT_E4M3 || t == LMT_E5M2; }
bool is_id(int t) { return t == LMT_I32 || t == LMT_I64; }
unsigned size_of(int t) { return t == LMT_I64 ? 8u : t == LMT_F32 || t == LMT_I32 ? 4u : t == LMT_F16 || t == LMT_BF16 ? 2u : 1u; }
bool off(const void* p, unsigned alignment) { return ((uintptr_t)p & (alignment - 1u)) != 0; }

int launched(const char* what, hipError_t e) {
  return e == hipSuccess ? 0 : fail(LMT_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}
int workspace_error(const void* workspace, uint64_t given, uint64_t needed) {
  if (needed == 0) return 0;
  if (!workspace) return fail(LMT_ERR_NULL, "workspace is NULL");
  if (off(workspace, 16)) return fail(LMT_ERR_ALIGN, "workspace is not 16-byte aligned");
  if (given < needed) return fail(LMT_ERR_WORKSPACE, "workspace of %llu bytes, %llu needed", (unsigned long long)given, (unsigned long long)needed);
  return 0;
}

// Rows of heads, as an input or as what is written: then no two elements may have one place.
int heads_error(const char* name, const lmt_heads* x, int dtype, uint64_t rows, uint64_t heads, uint64_t size, bool written, lmt::Heads* to) {
  if (!x || !x->at) return fail(LMT_ERR_NULL, "%s is NULL", name);
  if (off(x->at, size_of(dtype))) return fail(LMT_ERR_ALIGN, "%s is not aligned to its element size", name);
  const uint64_t row = rows > 1 ? x->row : 0, head = heads > 1 ? x->head : 0;  // the strides of one row, or of one head, say nothing
  if (row > lmt::kMaxStride || head > (1ull << 46)) return fail(LMT_ERR_LIMIT, "%s: a stride is too large", name);
  if (written) {
    const bool rows_inside = heads <= 1 || (rows > 1 && row < head);
    const uint64_t small = rows_inside ? row : head, count = rows_inside ? rows : heads, large = rows_inside ? head : row, of_large = rows_inside ? heads : rows;
    if ((count > 1 && small < size) || (of_large > 1 && large < (count - 1) * small + size)) return fail(LMT_ERR_ARG, "%s: elements have one place", name);
  }
  *to = {x->at, row, head};
  return 0;
}

int attend_error(const lmt_attend* a) {
  if (!a) return fail(LMT_ERR_NULL, "what attention goes by is NULL");
  if (a->dtype != LMT_F16 && a->dtype != LMT_BF16) return fail(LMT_ERR_ARG, "attention takes fp16 or bf16");
  if (a->flags & ~LMT_CAUSAL) return fail(LMT_ERR_ARG, "unknown flags");
  if (a->prefixes && !(a->flags & LMT_CAUSAL)) return fail(LMT_ERR_ARG, "prefixes without LMT_CAUSAL");
  if (!std::isfinite((float)a->scale)) return fail(LMT_ERR_ARG, "scale is not a finite fp32 number");
  if (!std::isfinite((float)a->cap) || a->cap < 0 || (a->cap != 0 && (float)a->cap < 1e-30f)) return fail(LMT_ERR_ARG, "cap is neither 0 nor a positive fp32 number");
  if (!std::isfinite((float)a->scale * 1.5f) || !std::isfinite((float)a->cap * 1.5f) || (a->cap != 0 && !std::isfinite((float)a->scale / (float)a->cap)))
    return fail(LMT_ERR_ARG, "scale, cap or scale / cap in units of log 2 are beyond fp32");
  if (a->rows > LMT_MAX_ROWS || a->sequences > LMT_MAX_ROWS || a->heads > LMT_MAX_HEADS || a->kv_heads > LMT_MAX_HEADS || a->size > LMT_MAX_HEAD)
    return fail(LMT_ERR_LIMIT, "sizes exceed LMT_MAX_ROWS, LMT_MAX_HEADS or LMT_MAX_HEAD");
  if (a->kv_heads == 0 ? a->heads != 0 : a->heads == 0 || a->heads % a->kv_heads != 0) return fail(LMT_ERR_ARG, "the query heads are no multiple of the key heads");
  if (lmt::attention_launches(a->rows, a->heads) > lmt::kMaxWorkgroups) return fail(LMT_ERR_LIMIT, "rows times heads are more than a launch can have");
  if (a->sequences != 0 && !a->starts) return fail(LMT_ERR_NULL, "starts is NULL");
  if (off(a->starts, 4) || off(a->lengths, 4) || off(a->prefixes, 4) || off(a->slopes, 4) || off(a->status, 4)) return fail(LMT_ERR_ALIGN, "a pointer is not aligned to its element size");
  return 0;
}
lmt::Attention attention_of(const lmt_attend& a) {
  lmt::Attention p = {};
  p.starts = a.starts, p.lengths = a.lengths, p.prefixes = a.prefixes, p.slopes = a.slopes, p.status = a.status;
  p.rows = (uint32_t)a.rows, p.heads = (uint32_t)a.heads, p.kv_heads = (uint32_t)a.kv_heads, p.group = (uint32_t)(a.heads / a.kv_heads), p.size = (uint32_t)a.size;
  p.sequences = (uint32_t)a.sequences, p.scale = (float)a.scale, p.cap = (float)a.cap, p.causal = (a.flags & LMT_CAUSAL) != 0;
  return p;
}

}  // namespace

extern "C" {

const char* lmt_last_error(void) { return g_error; }

uint64_t lmt_fp8_row_bytes(uint64_t cols) { return lmt::fp8_row_bytes(cols); }
uint64_t lmt_scale_row_bytes(uint64_t cols) { return lmt::scale_row_bytes(cols); }
uint64_t lmt_embed_grad_workspace(uint64_t n_tokens, uint64_t vocab, uint64_t width) { return lmt::embed_grad_workspace(n_tokens, vocab, width); }
uint64_t lmt_matmul_workspace(uint64_t m, uint64_t n, uint64_t k) { return lmt::matmul_workspace(m, n, k); }

int lmt_embed(const void* table, int table_dtype, uint64_t vocab, uint64_t width, uint64_t table_ld, const void* tokens, int token_dtype,
              uint64_t n_tokens, double scale, void* out, int out_dtype, uint64_t out_ld, int32_t* status, void* stream) {
  if (!is_float(table_dtype) || !is_float(out_dtype)) return fail(LMT_ERR_ARG, "table and out must be fp32, fp16 or bf16");
  if (!is_id(token_dtype)) return fail(LMT_ERR_ARG, "tokens must be LMT_I32 or LMT_I64");
  if (!std::isfinite((float)scale)) return fail(LMT_ERR_ARG, "scale is not a finite fp32 number");
  if (vocab > LMT_MAX_ROWS || n_tokens > LMT_MAX_ROWS || width > LMT_MAX_WIDTH) return fail(LMT_ERR_LIMIT, "sizes exceed LMT_MAX_ROWS or LMT_MAX_WIDTH");
  if (table_ld < width || out_ld < width) return fail(LMT_ERR_ARG, "a row stride is below width");
  if (n_tokens == 0 || width == 0) return 0;
  if ((!table && vocab != 0) || !tokens || !out) return fail(LMT_ERR_NULL, "table, tokens or out is NULL");
  if (off(table, size_of(table_dtype)) || off(out, size_of(out_dtype)) || off(tokens, size_of(token_dtype)) || off(status, 4))
    return fail(LMT_ERR_ALIGN, "a pointer is not aligned to its element size");
  const lmt::Embed p{table, tokens, out, table_ld, out_ld, (uint32_t)vocab, (uint32_t)width, (uint32_t)n_tokens, (float)scale, status};
  return launched("launching the lookup", lmt::launch_embed(p, table_dtype, token_dtype, out_dtype, (hipStream_t)stream));
}

int lmt_embed_grad(const void* grad_out, int grad_out_dtype, uint64_t grad_out_ld, const void* tokens, int token_dtype, uint64_t n_tokens,
                   double scale, int64_t skip_token, void* grad, int grad_dtype, uint64_t vocab, uint64_t width, uint64_t grad_ld,
                   uint32_t flags, int32_t* status, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!is_float(grad_out_dtype) || !is_float(grad_dtype)) return fail(LMT_ERR_ARG, "grad_out and grad must be fp32, fp16 or bf16");
  if (!is_id(token_dtype)) return fail(LMT_ERR_ARG, "tokens must be LMT_I32 or LMT_I64");
  if (flags & ~LMT_ACCUMULATE) return fail(LMT_ERR_ARG, "unknown flags");
  if (!std::isfinite((float)scale)) return fail(LMT_ERR_ARG, "scale is not a finite fp32 number");
  if (vocab > LMT_MAX_ROWS || n_tokens > LMT_MAX_ROWS || width > LMT_MAX_WIDTH) return fail(LMT_ERR_LIMIT, "sizes exceed LMT_MAX_ROWS or LMT_MAX_WIDTH");
  if (grad_out_ld < width || grad_ld < width) return fail(LMT_ERR_ARG, "a row stride is below width");
  const bool accumulate = (flags & LMT_ACCUMULATE) != 0;
  if (vocab == 0 || width == 0 || (n_tokens == 0 && accumulate)) return 0;
  if (!grad || (n_tokens != 0 && (!grad_out || !tokens))) return fail(LMT_ERR_NULL, "grad_out, tokens or grad is NULL");
  if (off(grad_out, size_of(grad_out_dtype)) || off(grad, size_of(grad_dtype)) || off(tokens, size_of(token_dtype)) || off(status, 4))
    return fail(LMT_ERR_ALIGN, "a pointer is not aligned to its element size");
  if (const int rc = workspace_error(workspace, workspace_bytes, lmt::embed_grad_workspace(n_tokens, vocab, width))) return rc;
  const lmt::EmbedGrad p{grad_out, tokens, grad, grad_out_ld, grad_ld, (uint32_t)vocab, (uint32_t)width, (uint32_t)n_tokens, (float)scale, skip_token, accumulate, status};
  return launched("launching the table's gradient", lmt::launch_embed_grad(p, grad_out_dtype, token_dtype, grad_dtype, workspace, (hipStream_t)stream));
}

int lmt_quantize(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int fp8, uint32_t flags, void* q, uint8_t* scales,
                 void* qt, uint8_t* scales_t, void* stream) {
  if (!is_float(dtype)) return fail(LMT_ERR_ARG, "x must be fp32, fp16 or bf16");
  if (!is_fp8(fp8)) return fail(LMT_ERR_ARG, "fp8 must be LMT_E4M3 or LMT_E5M2");
  if (flags & ~LMT_TILE_SCALES) return fail(LMT_ERR_ARG, "unknown flags");
  if (rows > LMT_MAX_ROWS || cols > LMT_MAX_WIDTH || (qt && rows > LMT_MAX_WIDTH)) return fail(LMT_ERR_LIMIT, "sizes exceed LMT_MAX_ROWS or LMT_MAX_WIDTH");
  if (ld < cols) return fail(LMT_ERR_ARG, "ld is below cols");
  if (!q != !scales || !qt != !scales_t) return fail(LMT_ERR_NULL, "a matrix without its scales, or scales without their matrix");
  if (rows == 0 || cols == 0) return 0;
  if (!q && !qt) return fail(LMT_ERR_NULL, "neither q nor qt is given");
  if (!x) return fail(LMT_ERR_NULL, "x is NULL");
  if (off(x, size_of(dtype)) || off(q, 16) || off(qt, 16)) return fail(LMT_ERR_ALIGN, "x is not aligned to its element size, or q or qt to 16 bytes");
  const lmt::Quantize p{x, ld, (uint32_t)rows, (uint32_t)cols, static_cast<uint8_t*>(q), scales, static_cast<uint8_t*>(qt), scales_t};
  return launched("launching the quantisation", lmt::launch_quantize(p, dtype, fp8, (flags & LMT_TILE_SCALES) != 0, (hipStream_t)stream));
}

int lmt_matmul(const void* a, int a_fp8, const uint8_t* a_scales, const void* b, int b_fp8, const uint8_t* b_scales, uint64_t m, uint64_t n,
               uint64_t k, void* c, int c_dtype, uint64_t ldc, uint32_t flags, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!is_fp8(a_fp8) || !is_fp8(b_fp8)) return fail(LMT_ERR_ARG, "a and b must be LMT_E4M3 or LMT_E5M2");
  if (!is_float(c_dtype)) return fail(LMT_ERR_ARG, "c must be fp32, fp16 or bf16");
  if (flags & ~(LMT_ACCUMULATE | LMT_FP32_SUMS)) return fail(LMT_ERR_ARG, "unknown flags");
  if (m > LMT_MAX_ROWS || n > LMT_MAX_ROWS || k > LMT_MAX_WIDTH) return fail(LMT_ERR_LIMIT, "sizes exceed LMT_MAX_ROWS or LMT_MAX_WIDTH");
  if (ldc < n) return fail(LMT_ERR_ARG, "ldc is below n");
  const bool accumulate = (flags & LMT_ACCUMULATE) != 0;
  if (m == 0 || n == 0 || (k == 0 && accumulate)) return 0;
  if (!c || (k != 0 && (!a || !a_scales || !b || !b_scales))) return fail(LMT_ERR_NULL, "an operand, its scales or c is NULL");
  if (off(a, 16) || off(b, 16) || off(a_scales, 4) || off(b_scales, 4) || off(c, size_of(c_dtype)))
    return fail(LMT_ERR_ALIGN, "operands must start on 16 bytes, scales on 4, c on its element size");
  if (const int rc = workspace_error(workspace, workspace_bytes, lmt::matmul_workspace(m, n, k))) return rc;
  const lmt::Matmul p{static_cast<const uint8_t*>(a), a_scales, static_cast<const uint8_t*>(b), b_scales, c, ldc, (uint32_t)m, (uint32_t)n, (uint32_t)k, accumulate,
                      (flags & LMT_FP32_SUMS) != 0, static_cast<float*>(workspace)};
  return launched("launching the product", lmt::launch_matmul(p, a_fp8, b_fp8, c_dtype, (hipStream_t)stream));
}

int lmt_cross_entropy(const void* logits, int dtype, uint64_t rows, uint64_t classes, uint64_t ld, const void* targets, int target_dtype,
                      int64_t ignore, const float* weights, float* loss, float* lse, void* grad, uint64_t grad_ld, int32_t* status, void* stream) {
  if (!is_float(dtype)) return fail(LMT_ERR_ARG, "logits must be fp32, fp16 or bf16");
  if (!is_id(target_dtype)) return fail(LMT_ERR_ARG, "targets must be LMT_I32 or LMT_I64");
  if (rows > LMT_MAX_ROWS || classes > LMT_MAX_ROWS) return fail(LMT_ERR_LIMIT, "sizes exceed LMT_MAX_ROWS");
  if (ld < classes || (grad && grad_ld < classes)) return fail(LMT_ERR_ARG, "a row stride is below classes");
  if (grad == logits && grad && grad_ld != ld) return fail(LMT_ERR_ARG, "a gradient in the logits' place must have their stride");
  if (rows == 0) return 0;
  if (classes == 0) return fail(LMT_ERR_ARG, "rows without classes");
  if (!logits || !targets) return fail(LMT_ERR_NULL, "logits or targets is NULL");
  if (off(logits, size_of(dtype)) || off(grad, size_of(dtype)) || off(targets, size_of(target_dtype)) || off(weights, 4) || off(loss, 4) || off(lse, 4) || off(status, 4))
    return fail(LMT_ERR_ALIGN, "a pointer is not aligned to its element size");
  const lmt::CrossEntropy p{logits, targets, weights, loss, lse, grad, ld, grad_ld, (uint32_t)rows, (uint32_t)classes, 0, ignore, status};
  return launched("launching the loss", lmt::launch_cross_entropy(p, dtype, target_dtype, (hipStream_t)stream));
}

uint64_t lmt_linear_cross_entropy_workspace(uint64_t rows, uint64_t classes, uint64_t width, int gradients) {
  return rows > LMT_MAX_WIDTH || classes > LMT_MAX_WIDTH || width > LMT_MAX_WIDTH ? 0 : lmt::linear_loss_workspace(rows, classes, width, gradients != 0);
}

uint64_t lmt_linear_cross_entropy_workspace_of(int dtype, uint64_t rows, uint64_t classes, uint64_t width, int gradients) {
  return (dtype != LMT_F16 && dtype != LMT_BF16) || rows > LMT_MAX_WIDTH || classes > LMT_MAX_WIDTH || width > LMT_MAX_WIDTH ? 0 : lmt::linear_loss_workspace_of(dtype, rows, classes, width, gradients != 0);
}

int lmt_linear_cross_entropy(const void* x, uint64_t x_ld, const void* table, uint64_t table_ld, int dtype, uint64_t rows, uint64_t classes,
                             uint64_t width, const void* targets, int target_dtype, int64_t ignore, const float* weights, float* loss, float* lse,
                             void* grad_x, uint64_t grad_x_ld, void* grad_table, int grad_table_dtype, uint64_t grad_table_ld, uint32_t flags,
                             int32_t* status, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (dtype != LMT_F16 && dtype != LMT_BF16) return fail(LMT_ERR_ARG, "x and table must be fp16 or bf16");
  if (!is_id(target_dtype)) return fail(LMT_ERR_ARG, "targets must be LMT_I32 or LMT_I64");
  if (grad_table && grad_table_dtype != dtype && grad_table_dtype != LMT_F32) return fail(LMT_ERR_ARG, "grad_table must be of the table's type or fp32");
  if (flags & ~LMT_ACCUMULATE) return fail(LMT_ERR_ARG, "unknown flags");
  if (rows > LMT_MAX_WIDTH || classes > LMT_MAX_WIDTH || width > LMT_MAX_WIDTH) return fail(LMT_ERR_LIMIT, "sizes exceed LMT_MAX_WIDTH");
  const auto tiles = [](uint64_t a, uint64_t b) { return lmt::ceil_div(a, 64) * lmt::ceil_div(b, 64); };
  if (tiles(rows, classes) > lmt::kMaxWorkgroups || tiles(rows, width) + tiles(classes, width) > lmt::kMaxWorkgroups)
    return fail(LMT_ERR_LIMIT, "rows times classes, or times width, are more than a launch can have");
  if (x_ld < width || table_ld < width || (grad_x && grad_x_ld < width) || (grad_table && grad_table_ld < width)) return fail(LMT_ERR_ARG, "a row stride is below width");
  if (rows == 0) {  // no row has a part in the table's gradient
    if (grad_table && !(flags & LMT_ACCUMULATE) && classes != 0 && width != 0) return fail(LMT_ERR_ARG, "no rows: a gradient of the table that is not added to would have to be cleared");
    return 0;
  }
  if (classes == 0 || width == 0) return fail(LMT_ERR_ARG, "rows without classes or elements");
  if (!x || !table || !targets) return fail(LMT_ERR_NULL, "x, table or targets is NULL");
  if (off(x, 2) || off(table, 2) || off(grad_x, 2) || off(grad_table, size_of(grad_table_dtype)) || off(targets, size_of(target_dtype)) || off(weights, 4) || off(loss, 4) ||
      off(lse, 4) || off(status, 4))
    return fail(LMT_ERR_ALIGN, "a pointer is not aligned to its element size");
  const lmt::LinearLoss p{x, table, targets, weights, loss, lse, grad_x, grad_table, workspace, x_ld, table_ld, grad_x_ld, grad_table_ld, (uint32_t)rows, (uint32_t)classes,
                          (uint32_t)width, target_dtype == LMT_I64, (flags & LMT_ACCUMULATE) != 0, grad_table && grad_table_dtype == LMT_F32, ignore, status};
  if (const int rc = workspace_error(workspace, workspace_bytes, lmt::linear_loss_workspace(p, dtype))) return rc;
  return launched("launching the loss", lmt::launch_linear_loss(p, dtype, (hipStream_t)stream));
}

int lmt_rotary(const lmt_heads* x, int dtype, uint64_t rows, uint64_t heads, uint64_t size, const void* positions, int position_dtype,
               const float* frequencies, uint64_t pairs, double magnitude, uint32_t flags, const lmt_heads* out, void* stream) {
  if (!is_float(dtype)) return fail(LMT_ERR_ARG, "x must be fp32, fp16 or bf16");
  if (!is_id(position_dtype)) return fail(LMT_ERR_ARG, "positions must be LMT_I32 or LMT_I64");
  if (flags & ~(LMT_NEIGHBOURS | LMT_INVERSE)) return fail(LMT_ERR_ARG, "unknown flags");
  if (!std::isfinite((float)magnitude)) return fail(LMT_ERR_ARG, "magnitude is not a finite fp32 number");
  if (rows > LMT_MAX_ROWS || heads > LMT_MAX_HEADS || size > LMT_MAX_HEAD) return fail(LMT_ERR_LIMIT, "sizes exceed LMT_MAX_ROWS, LMT_MAX_HEADS or LMT_MAX_HEAD");
  if (pairs > size / 2) return fail(LMT_ERR_ARG, "more pairs than a head has");
  if (rows == 0 || heads == 0 || size == 0) return 0;
  lmt::Rotary p = {};
  if (const int rc = heads_error("x", x, dtype, rows, heads, size, false, &p.x)) return rc;
  if (const int rc = heads_error("out", out, dtype, rows, heads, size, true, &p.out)) return rc;
  if (p.x.at == p.out.at && (p.x.row != p.out.row || p.x.head != p.out.head)) return fail(LMT_ERR_ARG, "out in x's place must have its strides");
  if (pairs != 0 && (!positions || !frequencies)) return fail(LMT_ERR_NULL, "positions or frequencies is NULL");
  if (off(positions, size_of(position_dtype)) || off(frequencies, 4)) return fail(LMT_ERR_ALIGN, "a pointer is not aligned to its element size");
  p.positions = positions, p.frequencies = frequencies, p.rows = (uint32_t)rows, p.heads = (uint32_t)heads, p.size = (uint32_t)size, p.pairs = (uint32_t)pairs;
  p.magnitude = (float)magnitude, p.neighbours = (flags & LMT_NEIGHBOURS) != 0, p.inverse = (flags & LMT_INVERSE) != 0;
  return launched("launching the rotary positions", lmt::launch_rotary(p, dtype, position_dtype, (hipStream_t)stream));
}

int lmt_attention(const lmt_attend* a, const lmt_heads* q, const lmt_heads* k, const lmt_heads* v, const lmt_heads* out, float* lse, void* stream) {
  if (const int rc = attend_error(a)) return rc;
  if (a->rows == 0 || a->heads == 0 || a->size == 0) return 0;
  lmt::Attention p = attention_of(*a);
  if (const int rc = heads_error("q", q, a->dtype, a->rows, a->heads, a->size, false, &p.q)) return rc;
  if (const int rc = heads_error("k", k, a->dtype, a->rows, a->kv_heads, a->size, false, &p.k)) return rc;
  if (const int rc = heads_error("v", v, a->dtype, a->rows, a->kv_heads, a->size, false, &p.v)) return rc;
  if (const int rc = heads_error("out", out, a->dtype, a->rows, a->heads, a->size, true, &p.out)) return rc;
  if (off(lse, 4)) return fail(LMT_ERR_ALIGN, "lse is not aligned to its element size");
  p.lse = lse;
  return launched("launching the attention", lmt::launch_attention(p, a->dtype, (hipStream_t)stream));
}

uint64_t lmt_attention_grad_workspace(uint64_t rows, uint64_t heads, uint64_t kv_heads, uint64_t size) {
  if (rows == 0 || heads == 0 || kv_heads == 0 || size == 0 || rows > LMT_MAX_ROWS || heads > LMT_MAX_HEADS || kv_heads > heads || size > LMT_MAX_HEAD) return 0;
  return lmt::attention_grad_workspace(rows, heads, kv_heads, size);
}

int lmt_attention_grad(const lmt_attend* a, const lmt_heads* grad_out, const lmt_heads* q, const lmt_heads* k, const lmt_heads* v, const lmt_heads* out,
                       const float* lse, const lmt_heads* grad_q, const lmt_heads* grad_k, const lmt_heads* grad_v, void* workspace, uint64_t workspace_bytes,
                       void* stream) {
  if (const int rc = attend_error(a)) return rc;
  if (a->rows == 0 || a->heads == 0 || a->size == 0) return 0;
  lmt::Attention p = attention_of(*a);
  const uint64_t rows = a->rows, heads = a->heads, kv_heads = a->kv_heads, size = a->size;
  if (const int rc = heads_error("grad_out", grad_out, a->dtype, rows, heads, size, false, &p.grad_out)) return rc;
  if (const int rc = heads_error("q", q, a->dtype, rows, heads, size, false, &p.q)) return rc;
  if (const int rc = heads_error("k", k, a->dtype, rows, kv_heads, size, false, &p.k)) return rc;
  if (const int rc = heads_error("v", v, a->dtype, rows, kv_heads, size, false, &p.v)) return rc;
  if (const int rc = heads_error("out", out, a->dtype, rows, heads, size, false, &p.out)) return rc;
  if (const int rc = heads_error("grad_q", grad_q, a->dtype, rows, heads, size, true, &p.grad_q)) return rc;
  if (const int rc = heads_error("grad_k", grad_k, a->dtype, rows, kv_heads, size, true, &p.grad_k)) return rc;
  if (const int rc = heads_error("grad_v", grad_v, a->dtype, rows, kv_heads, size, true, &p.grad_v)) return rc;
  if (!lse) return fail(LMT_ERR_NULL, "lse is NULL");
  if (off(lse, 4)) return fail(LMT_ERR_ALIGN, "lse is not aligned to its element size");
  if (const int rc = workspace_error(workspace, workspace_bytes, lmt::attention_grad_workspace(rows, heads, kv_heads, size))) return rc;
  p.lse = const_cast<float*>(lse);
  p.delta = static_cast<float*>(workspace), p.part = p.delta + lmt::round_up(rows * heads, 4), p.parts = lmt::attention_parts(rows, heads, kv_heads, size);
  return launched("launching the attention's gradient", lmt::launch_attention_grad(p, a->dtype, (hipStream_t)stream));
}

}  // extern "C"
