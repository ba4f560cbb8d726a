// Rotary positions (lmt.h): pairs of a head's elements turned by position * frequency.
#include "lmt_device.h"
#include "lmt_internal.h"

namespace lmt {
namespace {

constexpr uint32_t kThreads = 256, kTurns = 1024;  // kTurns: pairs of a workgroup's tokens

// Sine and cosine of position * frequency.  The product and its quarter turns are made in 64 bits: in 32 a position of a million
// would be off by a twentieth of a radian.  What is left of a quarter turn, at most half of one, is exact to 2^-26 of it in 32 bits.
__device__ __forceinline__ float2 turn_of(int64_t position, float frequency, float magnitude, bool inverse) {
  const double quarters = (double)position * (double)frequency * 0.63661977236758134308, whole = __builtin_rint(quarters);
  float s, c;
  sincospif(0.5f * (float)(quarters - whole), &s, &c);
  const int q = (int)(whole - 4.0 * __builtin_floor(0.25 * whole));
  const float sine = q & 1 ? c : s, cosine = q & 1 ? s : c;
  return {magnitude * (q == 1 || q == 2 ? -cosine : cosine), magnitude * ((q >= 2) != inverse ? -sine : sine)};
}

// A workgroup takes `tokens` rows: their turns go to LDS, made once for all heads, then `across` lanes (a power of two) take a head's pieces of 8
// elements: 8 pairs from two places or, NEIGHBOURS, 4 pairs in a row; behind them what is only copied.
// Memory bounds it: 32 768 rows of 32 heads of 64 in bf16 in 48 us, 5.6 TB/s.  (Streaming stores 59.6 -> 61 us among other calls and, where a batch stays in the Infinity Cache, 15.8 -> 24; streaming loads 63.)
template <typename T, typename I, bool NEIGHBOURS>
__global__ __launch_bounds__(kThreads) void k_rotary(const Rotary p, uint32_t tokens, uint32_t across, uint32_t pieces, uint32_t copies) {
  __shared__ float2 turns[kTurns];
  const uint32_t piece = threadIdx.x % across, step = kThreads / across;
  const uint32_t step_t = step / p.heads, step_h = step % p.heads;
  for (uint64_t block = blockIdx.x; block * tokens < p.rows; block += gridDim.x) {
    const uint32_t first = (uint32_t)(block * tokens), n = min(tokens, p.rows - first);
    __syncthreads();
    for (uint32_t x = threadIdx.x; x < n * p.pairs; x += kThreads) {
      const uint32_t t = x / p.pairs, f = x - t * p.pairs;
      turns[x] = turn_of(id_at<I>(p.positions, first + t), load1(p.frequencies + f), p.magnitude, p.inverse);
    }
    __syncthreads();
    uint32_t t = threadIdx.x / across / p.heads, h = threadIdx.x / across % p.heads;
    for (; t < n; t += step_t, h += step_h, t += h >= p.heads, h -= h >= p.heads ? p.heads : 0u) {
      const T* from = static_cast<const T*>(p.x.at) + (uint64_t)(first + t) * p.x.row + (uint64_t)h * p.x.head;
      T* to = static_cast<T*>(p.out.at) + (uint64_t)(first + t) * p.out.row + (uint64_t)h * p.out.head;
      const float2* turn = turns + t * p.pairs;
      for (uint32_t c = piece; c < pieces + copies; c += across) {
        if (c >= pieces) {  // the rest of the head
          const uint32_t at = 2u * p.pairs + (c - pieces) * 8u;
          Vec<T, 8> x;
          if (at + 8u <= p.size) load<false>(x, from + at), store<false>(to + at, x);
          else load_end(x, from + at, p.size - at, 0.f), store_end(to + at, x, p.size - at);
        } else if constexpr (NEIGHBOURS) {
          const uint32_t at = c * 8u, left = 2u * p.pairs - at;
          Vec<T, 8> x;
          if (left >= 8u) load<false>(x, from + at);
          else load_end(x, from + at, left, 0.f);
          float y[8];
#pragma unroll
          for (uint32_t e = 0; e < 4; ++e) {
            const float2 r = turn[min(c * 4u + e, p.pairs - 1u)];
            const float a = x.get(2 * e), b = x.get(2 * e + 1);
            y[2 * e] = __builtin_fmaf(a, r.x, -b * r.y), y[2 * e + 1] = __builtin_fmaf(a, r.y, b * r.x);
          }
          x.set(y);
          if (left >= 8u) store<false>(to + at, x);
          else store_end(to + at, x, left);
        } else {
          const uint32_t at = c * 8u, left = p.pairs - at;
          Vec<T, 8> x, y;
          if (left >= 8u) load<false>(x, from + at), load<false>(y, from + p.pairs + at);
          else load_end(x, from + at, left, 0.f), load_end(y, from + p.pairs + at, left, 0.f);
          float u[8], v[8];
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) {
            const float2 r = turn[min(at + e, p.pairs - 1u)];
            const float a = x.get(e), b = y.get(e);
            u[e] = __builtin_fmaf(a, r.x, -b * r.y), v[e] = __builtin_fmaf(a, r.y, b * r.x);
          }
          x.set(u), y.set(v);
          if (left >= 8u) store<false>(to + at, x), store<false>(to + p.pairs + at, y);
          else store_end(to + at, x, left), store_end(to + p.pairs + at, y, left);
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_rotary(const Rotary& p, int dtype, int position_dtype, hipStream_t s) {
  const uint32_t pieces = (uint32_t)ceil_div(p.neighbours ? 2 * p.pairs : p.pairs, 8), copies = p.x.at == p.out.at ? 0u : (uint32_t)ceil_div(p.size - 2 * p.pairs, 8);
  if (pieces + copies == 0) return hipSuccess;
  uint32_t across = 1;
  while (across < pieces + copies) across *= 2;
  // tokens: about eight items a thread, while there are two workgroups for every compute unit
  uint64_t tokens = std::min<uint64_t>(8 * kThreads / (across * p.heads), kTurns / std::max(1u, p.pairs));
  tokens = std::max<uint64_t>(1, std::min<uint64_t>(tokens, p.rows / (2 * kCus)));
  const uint32_t grid = (uint32_t)std::min<uint64_t>(ceil_div(p.rows, tokens), 1u << 22);
  const auto go = [&](auto t, auto i) {
    typedef decltype(t) T;
    typedef decltype(i) I;
    if (p.neighbours) hipLaunchKernelGGL((k_rotary<T, I, true>), dim3(grid), dim3(kThreads), 0, s, p, (uint32_t)tokens, across, pieces, copies);
    else hipLaunchKernelGGL((k_rotary<T, I, false>), dim3(grid), dim3(kThreads), 0, s, p, (uint32_t)tokens, across, pieces, copies);
    return hipGetLastError();
  };
  const auto typed = [&](auto t) { return position_dtype == LMT_I64 ? go(t, int64_t{}) : go(t, int32_t{}); };
  switch (dtype) {
    case LMT_F32: return typed(float{});
    case LMT_F16: return typed(_Float16{});
    default: return typed(bf16_t{});
  }
}

}  // namespace lmt
