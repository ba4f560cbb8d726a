// What the kernels of lmt.h share: element types as fp32 and back, accesses to tensors that may start anywhere.
#ifndef LMT_DEVICE_H_
#define LMT_DEVICE_H_

#include <hip/hip_runtime.h>

namespace lmt {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16_t;

// Tensor memory is reached through pointers that are explicitly global, so that loads are global_load with counted waits.
#define LMT_GLOBAL __attribute__((address_space(1)))

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(_Float16 x) { return (float)x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return __uint_as_float((uint32_t)__builtin_bit_cast(uint16_t, x) << 16); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) {
  return x;
}
template <>
__device__ __forceinline__ _Float16 from_f32<_Float16>(float x) {
  return (_Float16)x;
}
template <>
__device__ __forceinline__ bf16_t from_f32<bf16_t>(float x) {  // the hardware's conversion: nearest, ties to even, NaN stays NaN
  return (bf16_t)x;
}

// N consecutive elements, 4 to 32 bytes, at the alignment of one element: gfx950 runs in unaligned access mode, and told so
// the compiler emits the same wide accesses as for aligned data.
template <typename T, int N>
struct Vec {
  static constexpr int kWords = N * (int)sizeof(T) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) {
      return __uint_as_float(w[i]);
    } else {
      const uint16_t h = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
      return to_f32(__builtin_bit_cast(T, h));
    }
  }
  __device__ __forceinline__ void set(const float (&x)[N]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __float_as_uint(x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2)
        w[i / 2] = (uint32_t)__builtin_bit_cast(uint16_t, from_f32<T>(x[i])) |
                   (uint32_t)__builtin_bit_cast(uint16_t, from_f32<T>(x[i + 1])) << 16;
    }
  }
};
// One element, for rows that are shorter than a vector.
template <typename T>
struct Vec<T, 1> {
  T x;
  __device__ __forceinline__ float get(int) const { return to_f32(x); }
  __device__ __forceinline__ void set(const float (&f)[1]) { x = from_f32<T>(f[0]); }
};
template <int SIZE>
struct At;  // words aligned to elements of SIZE bytes
template <>
struct At<2> {
  typedef u32x4 x4 __attribute__((aligned(2)));
  typedef u32x2 x2 __attribute__((aligned(2)));
  typedef uint32_t x1 __attribute__((aligned(2)));
};
template <>
struct At<4> {
  typedef u32x4 x4 __attribute__((aligned(4)));
  typedef u32x2 x2 __attribute__((aligned(4)));
  typedef uint32_t x1;
};
template <bool NT, typename T, int N>
__device__ __forceinline__ void load_words(Vec<T, N>& v, const T* p) {
  constexpr int W = Vec<T, N>::kWords;
  static_assert(W == 1 || W == 2 || W % 4 == 0, "4, 8 or a multiple of 16 bytes");
  if constexpr (W == 1) {
    const LMT_GLOBAL auto* g = (const LMT_GLOBAL typename At<sizeof(T)>::x1*)p;
    if constexpr (NT) v.w[0] = __builtin_nontemporal_load(g);
    else v.w[0] = *g;
  } else if constexpr (W == 2) {
    const LMT_GLOBAL auto* g = (const LMT_GLOBAL typename At<sizeof(T)>::x2*)p;
    u32x2 x;
    if constexpr (NT) x = __builtin_nontemporal_load(g);
    else x = *g;
    v.w[0] = x.x, v.w[1] = x.y;
  } else {
    const LMT_GLOBAL auto* g = (const LMT_GLOBAL typename At<sizeof(T)>::x4*)p;
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      u32x4 x;
      if constexpr (NT) x = __builtin_nontemporal_load(g + i);
      else x = g[i];
      v.w[4 * i] = x.x, v.w[4 * i + 1] = x.y, v.w[4 * i + 2] = x.z, v.w[4 * i + 3] = x.w;
    }
  }
}
template <bool NT, typename T, int N>
__device__ __forceinline__ void store_words(T* p, const Vec<T, N>& v) {
  constexpr int W = Vec<T, N>::kWords;
  if constexpr (W == 1) {
    LMT_GLOBAL auto* g = (LMT_GLOBAL typename At<sizeof(T)>::x1*)p;
    if constexpr (NT) __builtin_nontemporal_store(v.w[0], g);
    else *g = v.w[0];
  } else if constexpr (W == 2) {
    LMT_GLOBAL auto* g = (LMT_GLOBAL typename At<sizeof(T)>::x2*)p;
    const u32x2 x = {v.w[0], v.w[1]};
    if constexpr (NT) __builtin_nontemporal_store(x, g);
    else *g = x;
  } else {
    LMT_GLOBAL auto* g = (LMT_GLOBAL typename At<sizeof(T)>::x4*)p;
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const u32x4 x = {v.w[4 * i], v.w[4 * i + 1], v.w[4 * i + 2], v.w[4 * i + 3]};
      if constexpr (NT) __builtin_nontemporal_store(x, g + i);
      else g[i] = x;
    }
  }
}
template <bool NT, typename T, int N>
__device__ __forceinline__ void load(Vec<T, N>& v, const T* p) {
  if constexpr (N == 1) {
    v.x = *(const LMT_GLOBAL T*)p;
  } else {
    load_words<NT>(v, p);
  }
}
template <bool NT, typename T, int N>
__device__ __forceinline__ void store(T* p, const Vec<T, N>& v) {
  if constexpr (N == 1) {
    *(LMT_GLOBAL T*)p = v.x;
  } else {
    store_words<NT>(p, v);
  }
}
template <typename T>
__device__ __forceinline__ T load1(const T* p) {
  return *(const LMT_GLOBAL T*)p;
}
template <typename T>
__device__ __forceinline__ void store1(T* p, T x) {
  *(LMT_GLOBAL T*)p = x;
}
// The first `n` < N elements (the end of a row); the others are `rest`, or are left alone.
template <typename T, int N>
__device__ __forceinline__ void load_end(Vec<T, N>& v, const T* p, uint32_t n, float rest) {
  float x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = (uint32_t)i < n ? to_f32(load1(p + i)) : rest;
  v.set(x);  // exact: the values are of this type
}
template <typename T, int N>
__device__ __forceinline__ void store_end(T* p, const Vec<T, N>& v, uint32_t n) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    if ((uint32_t)i < n) store1(p + i, from_f32<T>(v.get(i)));
}

// Ids (tokens, targets) of 32 or 64 bits.
template <typename I>
__device__ __forceinline__ int64_t id_at(const void* ids, uint64_t i) {
  return (int64_t)load1(static_cast<const I*>(ids) + i);
}

}  // namespace lmt
#endif  // LMT_DEVICE_H_
