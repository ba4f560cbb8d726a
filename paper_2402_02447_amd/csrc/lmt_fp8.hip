// 8-bit floating point with a power of two for every 128 elements: quantisation and products (lmt.h).
//
// The scales are powers of two because the matrix instructions of gfx950 take one for every 32 elements of an operand's row
// along with the operand (v_mfma_scale_f32_16x16x128_f8f6f4): with a block of 128 all four are the same byte, an
// instruction covers a block, and scaled blocks add up in the accumulators with no work beside it.
#include "lmt_device.h"
#include "lmt_internal.h"

namespace lmt {
namespace {

constexpr uint32_t kThreads = 256;
typedef int i32x8 __attribute__((ext_vector_type(8)));
template <int N>
struct Const {
  static constexpr int value = N;
};

// ---- quantisation ---------------------------------------------------------------------

// Magnitudes are compared as bits; infinities and NaN count as 0.
__device__ __forceinline__ uint32_t magnitude(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
// The biased exponent of a block's scale: the largest magnitude m 2^E (1 <= m < 2) goes to 1.75 * 2^top or below.
template <bool E5M2>
__device__ __forceinline__ uint32_t scale_of(uint32_t largest) {
  constexpr int top = E5M2 ? 15 : 8;
  const int e = (int)(largest >> 23) - top + ((largest & 0x7fffffu) > 0x600000u);
  return (uint32_t)max(e, 1);
}
__device__ __forceinline__ float inverse_of(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }
template <bool E5M2>
__device__ __forceinline__ uint32_t pack4(const float (&x)[4], float by) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool finite = (__float_as_uint(x[i]) & 0x7fffffffu) < 0x7f800000u;
    y[i] = finite ? x[i] * by : __builtin_nanf("");
  }
  int w = 0;
  if constexpr (E5M2) {
    w = __builtin_amdgcn_cvt_pk_bf8_f32(y[0], y[1], w, false);
    w = __builtin_amdgcn_cvt_pk_bf8_f32(y[2], y[3], w, true);
  } else {
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  }
  return (uint32_t)w;
}
// Largest over the 16 lanes of a row of lanes, in all of them.
__device__ __forceinline__ uint32_t max16(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));  // row_ror:8
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, false));
  return x;
}

// A workgroup takes squares of 128 x 128; a thread 8 rows of 8 columns, which it reads once for both results.
template <typename T, bool E5M2, bool TILE>
__global__ __launch_bounds__(kThreads) void k_quantize(const Quantize p, uint32_t tiles_across, uint32_t tiles_down) {
  __shared__ uint32_t col_max[4][128];
  __shared__ __align__(16) uint8_t turned[128 * 128];
  const uint32_t cg = threadIdx.x & 15u, rg = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const uint64_t q_row = round_up(p.cols, 128), s_row = 4 * ceil_div(p.cols, 512), qt_row = round_up(p.rows, 128), st_row = 4 * ceil_div(p.rows, 512);
  const uint64_t n_tiles = (uint64_t)tiles_across * tiles_down;
  for (uint64_t tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
    const uint32_t tr = (uint32_t)(tile / tiles_across), tc = (uint32_t)(tile % tiles_across);
    const uint32_t r0 = tr * 128u + rg * 8u, c0 = tc * 128u + cg * 8u;
    const uint32_t n = c0 < p.cols ? min(8u, p.cols - c0) : 0u;
    Vec<T, 8> x[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      x[j] = {};
      if (r0 + j < p.rows && n != 0) {
        const T* from = static_cast<const T*>(p.x) + (uint64_t)(r0 + j) * p.ld + c0;
        if (n == 8) load<false>(x[j], from);
        else load_end(x[j], from, n, 0.f);
      }
    }
    uint32_t row_max[8], cm[8] = {};
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      row_max[j] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t m = magnitude(x[j].get(i));
        row_max[j] = max(row_max[j], m);
        cm[i] = max(cm[i], m);
      }
    }
    uint32_t row_scale[8], col_scale[8];
    if constexpr (TILE) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, cm[i]);
      m = max16(m);
      m = max(m, (uint32_t)__shfl_xor((int)m, 16));
      m = max(m, (uint32_t)__shfl_xor((int)m, 32));
      if ((threadIdx.x & 63u) == 0) col_max[wave][0] = m;
      __syncthreads();
      m = max(max(col_max[0][0], col_max[1][0]), max(col_max[2][0], col_max[3][0]));
      const uint32_t s = scale_of<E5M2>(m);
#pragma unroll
      for (int i = 0; i < 8; ++i) row_scale[i] = col_scale[i] = s;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) row_scale[j] = scale_of<E5M2>(max16(row_max[j]));
      if (p.qt) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t m = max(cm[i], (uint32_t)__shfl_xor((int)cm[i], 16));
          m = max(m, (uint32_t)__shfl_xor((int)m, 32));
          if ((threadIdx.x & 48u) == 0) col_max[wave][cg * 8u + i] = m;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t c = cg * 8u + i;
          col_scale[i] = scale_of<E5M2>(max(max(col_max[0][c], col_max[1][c]), max(col_max[2][c], col_max[3][c])));
        }
      }
    }
    if (p.q) {
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j) {
        if (r0 + j >= p.rows) break;
        const float by = inverse_of(row_scale[j]);
        const float lo[4] = {x[j].get(0), x[j].get(1), x[j].get(2), x[j].get(3)}, hi[4] = {x[j].get(4), x[j].get(5), x[j].get(6), x[j].get(7)};
        const u32x2 w = {pack4<E5M2>(lo, by), pack4<E5M2>(hi, by)};
        *(LMT_GLOBAL u32x2*)(p.q + (uint64_t)(r0 + j) * q_row + c0) = w;
        if (cg == 0) {
          uint8_t* s = p.scales + (uint64_t)(r0 + j) * s_row;
          s[tc] = (uint8_t)row_scale[j];
          if (tc + 1u == tiles_across)
            for (uint64_t b = tc + 1u; b < s_row; ++b) s[b] = 127;
        }
      }
    }
    if (p.qt) {
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const float by = inverse_of(col_scale[i]);
        const float lo[4] = {x[0].get(i), x[1].get(i), x[2].get(i), x[3].get(i)}, hi[4] = {x[4].get(i), x[5].get(i), x[6].get(i), x[7].get(i)};
        const u32x2 w = {pack4<E5M2>(lo, by), pack4<E5M2>(hi, by)};
        // 16-byte pieces of a column's 128 bytes change places by the column's eight, so that they spread over the LDS banks
        *reinterpret_cast<u32x2*>(&turned[(cg * 8u + i) * 128u + ((rg / 2u) ^ (cg & 7u)) * 16u + (rg & 1u) * 8u]) = w;
        const uint32_t c = c0 + i;
        if (rg == 0 && c < p.cols) {
          uint8_t* s = p.scales_t + (uint64_t)c * st_row;
          s[tr] = (uint8_t)col_scale[i];
          if (tr + 1u == tiles_down)
            for (uint64_t b = tr + 1u; b < st_row; ++b) s[b] = 127;
        }
      }
      __syncthreads();
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) {
        const uint32_t c = k * 32u + threadIdx.x / 8u, piece = threadIdx.x & 7u;
        if (tc * 128u + c < p.cols)
          *(LMT_GLOBAL u32x4*)(p.qt + (uint64_t)(tc * 128u + c) * qt_row + (uint64_t)tr * 128u + piece * 16u) =
              *reinterpret_cast<const u32x4*>(&turned[c * 128u + (piece ^ (c / 8u & 7u)) * 16u]);
      }
    }
    __syncthreads();
  }
}

// ---- product ---------------------------------------------------------------------------

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A tile of c for WM x WN wavefronts, each with TM x TN squares of 32 x 32.  WIDE: operands are widened to bf16.
template <int WM_, int WN_, int TM_, int TN_>
struct Shape {
  static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_;
  static constexpr int waves = WM * WN, threads = 64 * waves;
  static constexpr int rows_m = 32 * TM * WM, rows_n = 32 * TN * WN;  // of c
  static constexpr int rows = rows_m + rows_n;                        // staged for every block of 128: a's, then b's
  static constexpr int loads = rows * 8 / threads;                    // of 16 bytes per thread
  static_assert(rows_m % (8 * waves) == 0 && rows_n % (8 * waves) == 0, "a load of all wavefronts is a's or b's");
};

// c's row i, columns j .. j + 3.
template <typename TC>
__device__ __forceinline__ void put4(const Matmul& p, uint32_t i, uint32_t j, const f32x4& d) {
  if (i >= p.m || j >= p.n) return;
  TC* to = static_cast<TC*>(p.c) + (uint64_t)i * p.ldc + j;
  const uint32_t n = min(4u, p.n - j);
  Vec<TC, 4> y = {};
  if (p.accumulate) {
    if (n == 4) load<false>(y, to);
    else load_end(y, to, n, 0.f);
  }
  float f[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) f[r] = p.accumulate ? d[r] + y.get(r) : d[r];
  y.set(f);
  if (n == 4) store<false>(to, y);
  else store_end(to, y, n);
}

// Which tile a workgroup has.
struct Tiles {
  uint32_t across, down, splits, split_blocks;  // of c in n and m; parts of k, and blocks of 128 in each
};
__device__ __forceinline__ void tile_of(const Tiles& t, uint32_t id, uint32_t* tm, uint32_t* tn, uint32_t* split) {
  const uint32_t n = t.across * t.down;
  *split = id / n, id %= n;
  *tm = id % t.down, *tn = id / t.down;
}

// The matrix instructions take X = b and Y = a: D[i][j] += sum over k of X[i][k] Y[j][k].  Lane l gives row l % 32 of both and has
// D[8 g + 4 (l / 32) + r][l % 32] in element 4 g + r: four neighbours of a row of c.  Which k a lane gives is of no concern as long
// as it is the same for X and Y.
template <typename S, int AF, int BF, bool WIDE>
__device__ __forceinline__ void step(f32x16 (&acc)[S::TM][S::TN], const uint8_t* a, const uint8_t* b, const uint32_t (&at)[2][2],
                                     const uint32_t (&as)[S::TM], const uint32_t (&bs)[S::TN], int block) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (!WIDE) {
      i32x8 x[S::TN], y[S::TM];
      const auto get = [&](const uint8_t* from) {
        const u32x4 lo = *reinterpret_cast<const u32x4*>(from + at[h][0]), hi = *reinterpret_cast<const u32x4*>(from + at[h][1]);
        return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
      };
#pragma unroll
      for (int f = 0; f < S::TN; ++f) x[f] = get(b + f * 4096);
#pragma unroll
      for (int f = 0; f < S::TM; ++f) y[f] = get(a + f * 4096);
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
          switch (block) {
            case 0: acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x[j], y[i], acc[i][j], BF, AF, 0, (int)bs[j], 0, (int)as[i]); break;
            case 1: acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x[j], y[i], acc[i][j], BF, AF, 1, (int)bs[j], 1, (int)as[i]); break;
            case 2: acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x[j], y[i], acc[i][j], BF, AF, 2, (int)bs[j], 2, (int)as[i]); break;
            default: acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x[j], y[i], acc[i][j], BF, AF, 3, (int)bs[j], 3, (int)as[i]); break;
          }
        }
    } else {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        bf16x8 x[S::TN][2], y[S::TM][2];
        const auto get = [&](bf16x8 (&to)[2], const uint8_t* from, uint32_t scales, auto e5m2) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(from + at[h][q]);
          const float s = __uint_as_float((scales >> (8 * block) & 255u) << 23);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            bf16x2 lo, hi;
            if constexpr (decltype(e5m2)::value) lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((int)w[v], s, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((int)w[v], s, true);
            else lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w[v], s, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w[v], s, true);
            to[v / 2][4 * (v % 2)] = lo.x, to[v / 2][4 * (v % 2) + 1] = lo.y;
            to[v / 2][4 * (v % 2) + 2] = hi.x, to[v / 2][4 * (v % 2) + 3] = hi.y;
          }
        };
#pragma unroll
        for (int f = 0; f < S::TN; ++f) get(x[f], b + f * 4096, bs[f], Const<BF>{});
#pragma unroll
        for (int f = 0; f < S::TM; ++f) get(y[f], a + f * 4096, as[f], Const<AF>{});
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
          for (int i = 0; i < S::TM; ++i)
#pragma unroll
            for (int j = 0; j < S::TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[j][v], y[i][v], acc[i][j], 0, 0, 0);
      }
    }
  }
}

template <typename S, int AF, int BF, bool WIDE, typename TC>
__global__ __launch_bounds__(S::threads, 2) void k_matmul(const Matmul p, const Tiles t) {
  __shared__ __align__(16) uint8_t stage[2][S::rows * 128];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, wm = wave / S::WN, wn = wave % S::WN;
  uint32_t tile_m, tile_n, split;
  tile_of(t, blockIdx.x, &tile_m, &tile_n, &split);
  const uint32_t m0 = tile_m * S::rows_m, n0 = tile_n * S::rows_n;
  const uint32_t blocks = (p.k + 127u) / 128u, s_row = (uint32_t)scale_row_bytes(p.k), row = blocks * 128u;
  const uint32_t first = split * t.split_blocks, end = min(blocks, first + t.split_blocks);
  // what this thread stages: rows behind the last one are the last one again.  The eight pieces of 16 bytes of a row's block change
  // places by the row, so that the lanes of a read of one piece from many rows spread over the LDS banks.
  const uint8_t *a0 = p.a + (uint64_t)m0 * row, *b0 = p.b + (uint64_t)n0 * row;
  const uint32_t last_m = p.m - 1u - m0, last_n = p.n - 1u - n0;
  uint32_t from[S::loads];
#pragma unroll
  for (int j = 0; j < S::loads; ++j) {
    const uint32_t r = (j * S::waves + wave) * 8u + lane / 8u;
    const uint32_t piece = ((lane & 7u) ^ (lane / 8u)) * 16u;
    from[j] = (j * S::waves * 8 < S::rows_m ? min(r, last_m) : min(r - S::rows_m, last_n)) * row + piece;
  }
  const auto fetch = [&](uint32_t block, int buffer) {
#pragma unroll
    for (int j = 0; j < S::loads; ++j) {
      const uint8_t* base = (j * S::waves * 8 < S::rows_m ? a0 : b0) + (uint64_t)block * 128u;
      __builtin_amdgcn_global_load_lds((const LMT_GLOBAL void*)(base + from[j]), (__attribute__((address_space(3))) void*)(&stage[buffer][(j * S::waves + wave) * 1024]), 16, 0, 0);
    }
  };
  // what this lane reads: pieces 4 h + 2 (l / 32) + q
  uint32_t at[2][2];
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) at[h][q] = (lane & 31u) * 128u + ((4u * h + 2u * (lane >> 5) + q) ^ (lane & 7u)) * 16u;
  const uint32_t a_at = wm * S::TM * 4096u, b_at = S::rows_m * 128u + wn * S::TN * 4096u;
  // scales of the lane's rows, four blocks at a time
  const uint8_t *as0 = p.a_scales + (uint64_t)m0 * s_row, *bs0 = p.b_scales + (uint64_t)n0 * s_row;
  uint32_t as_from[S::TM], bs_from[S::TN];
#pragma unroll
  for (int i = 0; i < S::TM; ++i) as_from[i] = min((wm * S::TM + i) * 32u + (lane & 31u), last_m) * s_row;
#pragma unroll
  for (int j = 0; j < S::TN; ++j) bs_from[j] = min((wn * S::TN + j) * 32u + (lane & 31u), last_n) * s_row;
  uint32_t as[S::TM], bs[S::TN], as_next[S::TM], bs_next[S::TN];
  const auto scales = [&](uint32_t block) {
#pragma unroll
    for (int i = 0; i < S::TM; ++i) as_next[i] = *(const LMT_GLOBAL uint32_t*)(as0 + block + as_from[i]);
#pragma unroll
    for (int j = 0; j < S::TN; ++j) bs_next[j] = *(const LMT_GLOBAL uint32_t*)(bs0 + block + bs_from[j]);
  };
  f32x16 acc[S::TM][S::TN] = {};
  if (first < end) {
    scales(first);
    fetch(first, 0);
  }
  for (uint32_t g = first; g < end; g += 4u) {
#pragma unroll
    for (int i = 0; i < S::TM; ++i) as[i] = as_next[i];
#pragma unroll
    for (int j = 0; j < S::TN; ++j) bs[j] = bs_next[j];
    if (g + 4u < end) scales(g + 4u);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (g + s >= end) break;
      __syncthreads();  // block g + s is staged, and nobody reads the other buffer any more
      if (g + s + 1u < end) fetch(g + s + 1u, (s + 1) & 1);
      step<S, AF, BF, WIDE>(acc, &stage[s & 1][a_at], &stage[s & 1][b_at], at, as, bs, s);
    }
  }
  float* part = t.splits > 1u ? p.workspace + ((uint64_t)blockIdx.x * S::threads + threadIdx.x) * 4u : nullptr;
#pragma unroll
  for (int i = 0; i < S::TM; ++i)
#pragma unroll
    for (int j = 0; j < S::TN; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 d = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        if (t.splits > 1u) {
          *(LMT_GLOBAL f32x4*)(part + (uint64_t)((i * S::TN + j) * 4 + g) * gridDim.x * S::threads * 4u) = d;
        } else {
          put4<TC>(p, m0 + (wm * S::TM + i) * 32u + (lane & 31u), n0 + (wn * S::TN + j) * 32u + g * 8u + (lane >> 5) * 4u, d);
        }
      }
}

// Adds the parts of k in order, one workgroup per tile and 4 x 64 x waves elements of it, in the layout of k_matmul's threads.
template <typename S, typename TC>
__global__ __launch_bounds__(S::threads) void k_matmul_join(const Matmul p, const Tiles t) {
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, wm = wave / S::WN, wn = wave % S::WN;
  const uint32_t n_tiles = t.across * t.down, piece = blockIdx.x / n_tiles, id = blockIdx.x % n_tiles;
  uint32_t tile_m, tile_n, split;
  tile_of(t, id, &tile_m, &tile_n, &split);
  const uint32_t i = piece / (S::TN * 4), j = piece / 4 % S::TN, g = piece % 4;
  const uint64_t split_size = (uint64_t)n_tiles * S::threads * 4u;
  const float* part = p.workspace + (uint64_t)piece * t.splits * split_size + ((uint64_t)id * S::threads + threadIdx.x) * 4u;
  f32x4 sum = *(const LMT_GLOBAL f32x4*)part;
  for (uint32_t s = 1; s < t.splits; ++s) sum += *(const LMT_GLOBAL f32x4*)(part + s * split_size);
  put4<TC>(p, tile_m * S::rows_m + (wm * S::TM + i) * 32u + (lane & 31u), tile_n * S::rows_n + (wn * S::TN + j) * 32u + g * 8u + (lane >> 5) * 4u, sum);
}

template <typename F>
hipError_t with_float(int dtype, F f) {
  switch (dtype) {
    case LMT_F32: return f(float{});
    case LMT_F16: return f(_Float16{});
    default: return f(bf16_t{});
  }
}
template <typename F>
hipError_t with_fp8(int fp8, F f) {
  return fp8 == LMT_E5M2 ? f(Const<1>{}) : f(Const<0>{});
}

}  // namespace

hipError_t launch_quantize(const Quantize& p, int dtype, int fp8, bool tile, hipStream_t s) {
  const uint32_t across = (uint32_t)ceil_div(p.cols, 128), down = (uint32_t)ceil_div(p.rows, 128);
  const uint32_t grid = (uint32_t)std::min<uint64_t>((uint64_t)across * down, 1u << 23);
  return with_float(dtype, [&](auto t) {
    return with_fp8(fp8, [&](auto f) {
      typedef decltype(t) T;
      constexpr bool E5M2 = decltype(f)::value == 1;
      if (tile) hipLaunchKernelGGL((k_quantize<T, E5M2, true>), dim3(grid), dim3(kThreads), 0, s, p, across, down);
      else hipLaunchKernelGGL((k_quantize<T, E5M2, false>), dim3(grid), dim3(kThreads), 0, s, p, across, down);
      return hipGetLastError();
    });
  });
}

namespace {

typedef Shape<2, 4, 4, 2> Large;   // 256 x 256
typedef Shape<2, 2, 2, 2> Medium;  // 128 x 128

struct Choice {
  bool large;
  Tiles tiles;
};
template <typename S>
Tiles tiles_of(uint64_t m, uint64_t n, uint64_t k, uint32_t splits) {
  const uint64_t blocks = ceil_div(k, 128);
  const uint64_t per = std::max<uint64_t>(4, round_up(ceil_div(blocks, splits), 4));
  return {(uint32_t)ceil_div(n, S::rows_n), (uint32_t)ceil_div(m, S::rows_m), (uint32_t)std::max<uint64_t>(1, ceil_div(blocks, per)), (uint32_t)per};
}
Choice choose(uint64_t m, uint64_t n, uint64_t k) {
  const uint64_t large = ceil_div(m, Large::rows_m) * ceil_div(n, Large::rows_n);
  const uint64_t medium = ceil_div(m, Medium::rows_m) * ceil_div(n, Medium::rows_n);
  if (large >= kCus) return {true, tiles_of<Large>(m, n, k, 1)};
  const uint64_t splits = std::min<uint64_t>(std::max<uint64_t>(1, kCus / large), std::max<uint64_t>(1, k / 2048));
  if (large * splits >= 128) return {true, tiles_of<Large>(m, n, k, (uint32_t)splits)};
  return {false, tiles_of<Medium>(m, n, k, (uint32_t)std::min<uint64_t>(std::max<uint64_t>(1, kCus / medium), std::max<uint64_t>(1, k / 1024)))};
}

}  // namespace

uint64_t matmul_workspace(uint64_t m, uint64_t n, uint64_t k) {
  if (m == 0 || n == 0) return 0;
  const Choice c = choose(m, n, k);
  const uint64_t tile = c.large ? Large::rows_m * Large::rows_n : Medium::rows_m * Medium::rows_n;
  return c.tiles.splits > 1 ? 4 * tile * c.tiles.splits * c.tiles.across * c.tiles.down : 0;
}

hipError_t launch_matmul(const Matmul& p, int a_fp8, int b_fp8, int c_dtype, hipStream_t s) {
  const Choice c = choose(p.m, p.n, p.k);
  const auto go = [&](auto shape, auto af, auto bf, auto tc) {
    typedef decltype(shape) S;
    typedef decltype(tc) TC;
    const uint32_t n_tiles = c.tiles.across * c.tiles.down;
    hipLaunchKernelGGL((k_matmul<S, decltype(af)::value, decltype(bf)::value, sizeof(TC) == 4, TC>), dim3(n_tiles * c.tiles.splits), dim3(S::threads), 0, s, p, c.tiles);
    if (c.tiles.splits > 1)
      hipLaunchKernelGGL((k_matmul_join<S, TC>), dim3(n_tiles * S::TM * S::TN * 4), dim3(S::threads), 0, s, p, c.tiles);
    return hipGetLastError();
  };
  return with_fp8(a_fp8, [&](auto af) {
    return with_fp8(b_fp8, [&](auto bf) {
      return with_float(c_dtype, [&](auto tc) { return c.large ? go(Large{}, af, bf, tc) : go(Medium{}, af, bf, tc); });
    });
  });
}

}  // namespace lmt
