// Between the argument checks (lmt.cpp) and the kernels' launches (lmt_embed.hip, lmt_fp8.hip, lmt_loss.hip, lmt_rotary.hip,
// lmt_attention.hip, lmt_linear_loss.hip) of lmt.h.
// Launchers take checked arguments, only enqueue, and return the last HIP error.
#ifndef LMT_INTERNAL_H_
#define LMT_INTERNAL_H_

#include <hip/hip_runtime.h>

#include <algorithm>

#include "lmt.h"

namespace lmt {

constexpr uint32_t kCus = 256;  // compute units of an MI355X, in 8 XCDs of 32

__host__ __device__ constexpr uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
__host__ __device__ constexpr uint64_t round_up(uint64_t a, uint64_t b) { return ceil_div(a, b) * b; }
__host__ __device__ constexpr uint64_t fp8_row_bytes(uint64_t cols) { return round_up(cols, 128); }
__host__ __device__ constexpr uint64_t scale_row_bytes(uint64_t cols) { return 4 * ceil_div(cols, 512); }

struct Embed {
  const void *table, *tokens;
  void* out;
  uint64_t table_ld, out_ld;
  uint32_t vocab, width, n_tokens;
  float scale;
  int32_t* status;
};
hipError_t launch_embed(const Embed& p, int table_dtype, int token_dtype, int out_dtype, hipStream_t s);

struct EmbedGrad {
  const void *grad_out, *tokens;
  void* grad;
  uint64_t grad_out_ld, grad_ld;
  uint32_t vocab, width, n_tokens;
  float scale;
  int64_t skip_token;
  bool accumulate;
  int32_t* status;
};
uint64_t embed_grad_workspace(uint64_t n_tokens, uint64_t vocab, uint64_t width);
hipError_t launch_embed_grad(const EmbedGrad& p, int grad_out_dtype, int token_dtype, int grad_dtype, void* workspace,
                             hipStream_t s);

struct Quantize {
  const void* x;
  uint64_t ld;
  uint32_t rows, cols;
  uint8_t *q, *scales, *qt, *scales_t;
};
hipError_t launch_quantize(const Quantize& p, int dtype, int fp8, bool tile, hipStream_t s);

struct Matmul {
  const uint8_t *a, *a_scales, *b, *b_scales;
  void* c;
  uint64_t ldc;
  uint32_t m, n, k;
  bool accumulate, fp32_sums;
  float* workspace;
};
uint64_t matmul_workspace(uint64_t m, uint64_t n, uint64_t k);
hipError_t launch_matmul(const Matmul& p, int a_fp8, int b_fp8, int c_dtype, hipStream_t s);

struct CrossEntropy {
  const void *logits, *targets;
  const float* weights;
  float *loss, *lse;
  void* grad;
  uint64_t ld, grad_ld;
  uint32_t rows, classes, first;  // first: the launch's first row
  int64_t ignore;
  int32_t* status;
};
hipError_t launch_cross_entropy(const CrossEntropy& p, int dtype, int target_dtype, hipStream_t s);

struct Heads {  // lmt_heads
  void* at;
  uint64_t row, head;
};

struct Rotary {
  Heads x, out;
  const void* positions;
  const float* frequencies;
  uint32_t rows, heads, size, pairs;
  float magnitude;
  bool neighbours, inverse;
};
hipError_t launch_rotary(const Rotary& p, int dtype, int position_dtype, hipStream_t s);

struct Attention {
  Heads q, k, v, out, grad_out, grad_q, grad_k, grad_v;
  float *lse, *delta, *part;  // delta: [heads][rows]; part: sums of parts of a key head's query heads
  const int32_t *starts, *lengths, *prefixes;
  const float* slopes;
  int32_t* status;
  uint32_t rows, heads, kv_heads, group, parts, size, sequences, cuts;  // group: query heads of a key head; cuts: sequences, where they cut blocks of rows
  float scale, cap;
  bool causal;
};
constexpr uint64_t kMaxStride = 0x7fffffffu;    // between rows, in elements
constexpr uint64_t kMaxWorkgroups = 0x7fffffu;  // of up to 512 threads: a launch has fewer than 2^32 threads
uint64_t attention_launches(uint64_t rows, uint64_t heads);  // workgroups of the largest launch
uint32_t attention_parts(uint64_t rows, uint64_t heads, uint64_t kv_heads, uint64_t size);
uint64_t attention_grad_workspace(uint64_t rows, uint64_t heads, uint64_t kv_heads, uint64_t size);
hipError_t launch_attention(const Attention& p, int dtype, hipStream_t s);
hipError_t launch_attention_grad(const Attention& p, int dtype, hipStream_t s);

struct LinearLoss {
  const void *x, *table, *targets;
  const float* weights;
  float *loss, *lse;
  void *grad_x, *grad_table, *workspace;
  uint64_t x_ld, table_ld, grad_x_ld, grad_table_ld;
  uint32_t rows, classes, width;
  bool wide_targets, accumulate, grad_table_f32;
  int64_t ignore;
  int32_t* status;
};
uint64_t linear_loss_workspace(uint64_t rows, uint64_t classes, uint64_t width, bool gradients);                // of any call
uint64_t linear_loss_workspace_of(int dtype, uint64_t rows, uint64_t classes, uint64_t width, bool gradients);  // of aligned ones
uint64_t linear_loss_workspace(const LinearLoss& p, int dtype);                                                // of this one
hipError_t launch_linear_loss(const LinearLoss& p, int dtype, hipStream_t s);

}  // namespace lmt
#endif  // LMT_INTERNAL_H_
