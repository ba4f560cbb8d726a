// Cross entropy of rows of logits with its gradient (lmt.h).
#include "lmt_device.h"
#include "lmt_internal.h"

namespace lmt {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr uint32_t kThreads = 256, kWaves = kThreads / 64;

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
// ... times c, with results below 2^-126 too, which the instruction cuts to 0.
__device__ __forceinline__ float scaled_term(float x, float top, float c) {
  return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f((x - top) * kLog2e + 32.f) * c, -32);
}

template <typename T, typename I>
__global__ __launch_bounds__(kThreads) void k_cross_entropy(const CrossEntropy p) {
  __shared__ float red[2][kWaves];
  constexpr int V = 16 / sizeof(T);
  for (uint64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(p.logits) + row * p.ld;
    const int64_t target = id_at<I>(p.targets, row);
    const bool there = target != p.ignore && (uint64_t)target < p.classes;
    if (threadIdx.x == 0 && target != p.ignore && !there && p.status) atomicOr(p.status, LMT_STATUS_BAD_TARGET);
    const float w = !there ? 0.f : p.weights ? p.weights[row] : 1.f;
    const uint32_t whole = p.classes / V;
    float top = -INFINITY;
    for (uint32_t i = threadIdx.x; i < whole; i += kThreads) {
      Vec<T, V> v;
      load<false>(v, x + (uint64_t)i * V);
#pragma unroll
      for (int j = 0; j < V; ++j) top = fmaxf(top, v.get(j));
    }
    for (uint32_t j = whole * V + threadIdx.x; j < p.classes; j += kThreads) top = fmaxf(top, to_f32(load1(x + j)));
    top = wave_max(top);
    if ((threadIdx.x & 63u) == 0) red[0][threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < kWaves; ++i) top = fmaxf(top, red[0][i]);
    const float from = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    for (uint32_t i = threadIdx.x; i < whole; i += kThreads) {
      Vec<T, V> v;
      load<false>(v, x + (uint64_t)i * V);
#pragma unroll
      for (int j = 0; j < V; ++j) sum += term(v.get(j), from);
    }
    for (uint32_t j = whole * V + threadIdx.x; j < p.classes; j += kThreads) sum += term(to_f32(load1(x + j)), from);
    sum = wave_sum(sum);
    if ((threadIdx.x & 63u) == 0) red[1][threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < kWaves; ++i) sum += red[1][i];
    if (threadIdx.x == 0) {
      const float lse = sum == 0.f ? -INFINITY : top + __logf(sum);
      if (p.lse) p.lse[row] = lse;
      if (p.loss) p.loss[row] = !there ? 0.f : sum == 0.f ? INFINITY : w * (lse - to_f32(load1(x + target)));
    }
    __syncthreads();  // the target's logit is read before a gradient in its place is written
    if (!p.grad) continue;
    T* g = static_cast<T*>(p.grad) + row * p.grad_ld;
    const bool zero = !there || sum == 0.f;  // 0: nothing but -Inf (the largest logit adds 1, NaN makes the sum NaN)
    const float c = w / sum;
    const auto grad = [&](float v, uint64_t j) {
      const float y = scaled_term(v, from, c);
      return zero ? 0.f : j == (uint64_t)target ? y - w : y;
    };
    for (uint32_t i = threadIdx.x; i < whole; i += kThreads) {
      Vec<T, V> v;
      float f[V];
      load<false>(v, x + (uint64_t)i * V);
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = grad(v.get(j), (uint64_t)i * V + j);
      v.set(f);
      store<false>(g + (uint64_t)i * V, v);
    }
    for (uint32_t j = whole * V + threadIdx.x; j < p.classes; j += kThreads) store1(g + j, from_f32<T>(grad(to_f32(load1(x + j)), j)));
  }
}

}  // namespace

hipError_t launch_cross_entropy(const CrossEntropy& p, int dtype, int target_dtype, hipStream_t s) {
  const dim3 grid(std::min(p.rows, 1u << 20)), block(kThreads);
  const auto go = [&](auto t, auto id) {
    hipLaunchKernelGGL((k_cross_entropy<decltype(t), decltype(id)>), grid, block, 0, s, p);
    return hipGetLastError();
  };
  const auto with = [&](auto id) { return dtype == LMT_F32 ? go(float{}, id) : dtype == LMT_F16 ? go(_Float16{}, id) : go(bf16_t{}, id); };
  return target_dtype == LMT_I64 ? with(int64_t{}) : with(int32_t{});
}

}  // namespace lmt
