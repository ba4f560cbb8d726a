// Cross entropy of rows of logits with its gradient (lmt.h).
//
// lse = top + log(sum of exp(x - top)), loss = w (lse - x[target]), grad = w (exp(x - top) / sum - [j = target]).  Bound by memory: a row
// is read once, kept in registers while its maximum and then its sum are found, and the gradient is written from there
// (3 sweeps over memory, the last two from cache: 562 us at 16 384 x 30 522 in bf16, this 328).  Rows longer
// than the registers of a workgroup are read twice, with a running maximum and sum the first time.
#include "lmt_device.h"
#include "lmt_internal.h"

namespace lmt {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) x += __shfl_xor(x, d);
  return x;
}

// exp(x - top) for x <= top.  The difference comes first: top * log2(e) alone would overflow where a row is masked with the
// type's lowest value.
__device__ __forceinline__ float term(float x, float top) { return __builtin_amdgcn_exp2f((x - top) * kLog2e); }
// ... times c, with results below 2^-126 too, which the instruction cuts to 0: as the square of the root, whose argument has the same bits (an offset to
// the exponent instead, taken off again behind, would hold an argument of 16 to 32 to 2^-20).
__device__ __forceinline__ float scaled_term(float x, float top, float c) {
  const float root = __builtin_amdgcn_exp2f((x - top) * (0.5f * kLog2e));
  return root * c * root;
}

// What a row has beside its logits.
struct Row {
  int64_t target;
  bool there;  // there is a target
  float w;
};
template <typename I>
__device__ __forceinline__ Row row_of(const CrossEntropy& p, uint64_t row, bool report) {
  Row r;
  r.target = id_at<I>(p.targets, row);
  r.there = r.target != p.ignore && (uint64_t)r.target < p.classes;
  if (report && p.status && !r.there && r.target != p.ignore) atomicOr(p.status, LMT_STATUS_BAD_TARGET);
  r.w = !r.there ? 0.f : p.weights ? load1(p.weights + row) : 1.f;
  return r;
}
// Sum 0: nothing but -Inf (the largest logit adds 1, NaN makes the sum NaN).  The loss is not made of lse, which is rounded to the size of the logits: a small
// loss would be the difference of two large numbers.
__device__ __forceinline__ void put_loss(const CrossEntropy& p, uint64_t row, const Row& r, float top, float sum, float at_target) {
  const float log_sum = __logf(sum);
  if (p.lse) p.lse[row] = sum == 0.f ? -INFINITY : top + log_sum;
  if (p.loss) p.loss[row] = !r.there ? 0.f : sum == 0.f ? INFINITY : r.w * ((top - at_target) + log_sum);
}

// One row per workgroup of THREADS threads (64: per wavefront), N vectors of 16 bytes per thread; what is left behind the last whole vector
// goes one element to a thread.  16 384 x 30 522 in bf16 (512 threads of 8 vectors) 328 us a call in a row of calls, 2.0 GB, 6.1 TB/s
// (under a kernel trace, which sets calls apart, 331 to 357; streaming stores of the gradient 353 in a row); in place 331, without gradient 172; 19 rows in fp32
// (1 024 threads of 8) 6.5, the latency of one row.
template <typename T, typename I, int THREADS, int N>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void k_cross_entropy(const CrossEntropy p) {
  constexpr int V = 16 / sizeof(T), kRowWaves = THREADS / 64;
  constexpr uint32_t kLowest = sizeof(T) == 4 ? 0xff800000u : __is_same(T, _Float16) ? 0xfc00fc00u : 0xff80ff80u;  // -Inf
  __shared__ float red[2][kRowWaves], goal;
  const uint32_t me = threadIdx.x % THREADS, wave = me >> 6;
  const uint64_t row = p.first + (THREADS < 256 ? (uint64_t)blockIdx.x * (256 / THREADS) + threadIdx.x / THREADS : blockIdx.x);
  if (row >= p.rows) return;
  const Row r = row_of<I>(p, row, me == 0);
  const bool read = r.there || p.lse;  // else nothing of the row counts
  const T* x = static_cast<const T*>(p.logits) + row * p.ld;
  const uint32_t whole = p.classes / V, left = p.classes - whole * V;
  Vec<T, V> v[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t i = k * THREADS + me;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[k].w[j] = kLowest;
    if (read && i < whole) load<true>(v[k], x + (uint64_t)i * V);
  }
  const float end = read && me < left ? to_f32(load1(x + (uint64_t)whole * V + me)) : -INFINITY;
  float at_target = r.there && me == 0 ? to_f32(load1(x + r.target)) : 0.f;
  float top = end;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) top = fmaxf(top, v[k].get(j));
  top = wave_max(top);
  if constexpr (kRowWaves > 1) {
    if ((me & 63u) == 0) red[0][wave] = top;
    if (me == 0) goal = at_target;  // has arrived before anyone writes a gradient in its place
    __syncthreads();
    at_target = goal;
#pragma unroll
    for (int i = 0; i < kRowWaves; ++i) top = fmaxf(top, red[0][i]);
  }
  if (top == -INFINITY) top = 0.f;
  float sum = term(end, top);
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) sum += term(v[k].get(j), top);
  sum = wave_sum(sum);
  if constexpr (kRowWaves > 1) {
    if ((me & 63u) == 0) red[1][wave] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < kRowWaves; ++i) sum += red[1][i];
  }
  if (me == 0) put_loss(p, row, r, top, sum, at_target);
  if (!p.grad) return;
  T* g = static_cast<T*>(p.grad) + row * p.grad_ld;
  const bool zero = !r.there || sum == 0.f;
  const float c = r.w / sum;
  // the target's element, of the vector and of those behind the last one that this thread has
  const uint32_t target = zero ? ~0u : (uint32_t)r.target;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t i = k * THREADS + me;
    float f[V];
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = zero ? 0.f : scaled_term(v[k].get(j), top, c);
    if (i == target / V) {
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] -= target % V == (uint32_t)j ? r.w : 0.f;
    }
    v[k].set(f);
    if (i < whole) store<false>(g + (uint64_t)i * V, v[k]);
  }
  if (me < left) {
    const uint32_t j = whole * V + me;
    const float f = zero ? 0.f : scaled_term(end, top, c);
    store1(g + j, from_f32<T>(j == target ? f - r.w : f));
  }
}

// Rows of any length: a running maximum and sum per thread, joined at the end; then the gradient from a second reading.
// 512 x 262 144 in bf16: 149 us (805 MB, 5.4 TB/s).
constexpr int kLongThreads = 1024, kLongWaves = kLongThreads / 64;
template <typename T, typename I>
__global__ __launch_bounds__(kLongThreads) void k_cross_entropy_long(const CrossEntropy p) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float red[2][kLongWaves], goal;
  const uint32_t me = threadIdx.x;
  const uint64_t row = (uint64_t)p.first + blockIdx.x;
  const Row r = row_of<I>(p, row, me == 0);
  const T* x = static_cast<const T*>(p.logits) + row * p.ld;
  const uint32_t whole = p.classes / V, left = p.classes - whole * V;
  const float end = me < left ? to_f32(load1(x + (uint64_t)whole * V + me)) : -INFINITY;
  float top = end, sum = end == -INFINITY ? 0.f : term(end, end);
  constexpr int kAhead = 4;
  for (uint32_t i0 = me; i0 < whole; i0 += kAhead * kLongThreads) {
    Vec<T, V> v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) load<false>(v[k], x + (uint64_t)min(i0 + k * kLongThreads, whole - 1u) * V);
    float now = top;
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) now = fmaxf(now, v[k].get(j));
    const float base = now == -INFINITY ? 0.f : now;
    sum = sum == 0.f ? 0.f : sum * term(top, base);
    top = now;
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i0 + k * kLongThreads < whole) {
#pragma unroll
        for (int j = 0; j < V; ++j) sum += term(v[k].get(j), base);
      }
  }
  const float mine = top;
  top = wave_max(top);
  if ((me & 63u) == 0) red[0][me >> 6] = top;
  if (me == 0) goal = r.there ? to_f32(load1(x + r.target)) : 0.f;  // has arrived before anyone writes a gradient in its place
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kLongWaves; ++i) top = fmaxf(top, red[0][i]);
  if (top == -INFINITY) top = 0.f;
  sum = wave_sum(sum == 0.f ? 0.f : sum * term(mine, top));
  if ((me & 63u) == 0) red[1][me >> 6] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < kLongWaves; ++i) sum += red[1][i];
  if (me == 0) put_loss(p, row, r, top, sum, goal);
  if (!p.grad) return;
  T* g = static_cast<T*>(p.grad) + row * p.grad_ld;
  const bool zero = !r.there || sum == 0.f;
  const float c = r.w / sum;
  const uint32_t target = zero ? ~0u : (uint32_t)r.target;
#pragma unroll 4
  for (uint32_t i = me; i < whole; i += kLongThreads) {
    Vec<T, V> v;
    float f[V];
    load<false>(v, x + (uint64_t)i * V);
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = zero ? 0.f : scaled_term(v.get(j), top, c);
    if (i == target / V) {
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] -= target % V == (uint32_t)j ? r.w : 0.f;
    }
    v.set(f);
    store<false>(g + (uint64_t)i * V, v);
  }
  if (me < left) {
    const uint32_t j = whole * V + me;
    const float f = zero ? 0.f : scaled_term(end, top, c);
    store1(g + j, from_f32<T>(j == target ? f - r.w : f));
  }
}

}  // namespace

hipError_t launch_cross_entropy(const CrossEntropy& p, int dtype, int target_dtype, hipStream_t s) {
  const auto go = [&](auto t, auto id) {
    typedef decltype(t) T;
    typedef decltype(id) I;
    const uint32_t whole = p.classes / (16 / sizeof(T));  // vectors of a row
    const auto launch = [&](void (*kernel)(const CrossEntropy), uint32_t rows_each, int threads) {
      constexpr uint64_t kMost = 1u << 21;  // workgroups to a launch: 32 bits count the threads of one
      CrossEntropy part = p;
      for (uint64_t first = 0; first < p.rows; first += kMost * rows_each) {
        part.first = (uint32_t)first;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)std::min(kMost, ceil_div(p.rows - first, rows_each))), dim3(threads), 0, s, part);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      }
      return hipSuccess;
    };
    // The fewest threads that hold a row in a few vectors each: more of them leave lanes without work and rows waiting for each other.  bf16, us:
    // 100 000 x 100 by 64 threads 55 (by 256: 166), 20 000 x 1 000 by 64 18.6 (256: 40), 8 000 x 8 000 by 256 43 (512: 57), 8 192 x 30 522
    // by 512 170 (1 024: 338), 20 rows of that length 6.5 (9.1).
    if (whole <= 64 * 2) return launch(k_cross_entropy<T, I, 64, 2>, 4, 256);
    if (whole <= 256 * 2) return launch(k_cross_entropy<T, I, 256, 2>, 1, 256);
    if (whole <= 256 * 4) return launch(k_cross_entropy<T, I, 256, 4>, 1, 256);
    if (whole <= 512 * 4) return launch(k_cross_entropy<T, I, 512, 4>, 1, 512);
    if (whole <= 512 * 8) return launch(k_cross_entropy<T, I, 512, 8>, 1, 512);
    if (whole <= 1024 * 8) return launch(k_cross_entropy<T, I, 1024, 8>, 1, 1024);
    if (whole <= 1024 * 16) return launch(k_cross_entropy<T, I, 1024, 16>, 1, 1024);
    return launch(k_cross_entropy_long<T, I>, 1, kLongThreads);
  };
  const auto with = [&](auto id) { return dtype == LMT_F32 ? go(float{}, id) : dtype == LMT_F16 ? go(_Float16{}, id) : go(bf16_t{}, id); };
  return target_dtype == LMT_I64 ? with(int64_t{}) : with(int32_t{});
}

}  // namespace lmt
