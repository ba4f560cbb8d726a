// 8-bit floating point with a power of two for every 128 elements: quantisation and products (lmt.h).
//
// c[i][j] = sum over blocks of 2^(ea + eb) times the sum over the block of a b.  The scales are powers of two because the matrix
// instructions of gfx950 take one for every 32 elements of an operand's row along with the operand
// (v_mfma_scale_f32_32x32x64_f8f6f4): with a block of 128 all four are the same byte, and scaled blocks add up in the accumulators
// with no work beside it.
// Those instructions line up the products of eight neighbours before they add them, on a grid that the largest of them sets; what lies below it is cut off.
// Measured, of a result's 2-norm and whatever k: 1.5e-5 on normal numbers in e4m3 (e5m2 9e-6), up to 4e-5 where magnitudes spread over
// e^2, a drift of 3e-6 towards zero where all terms have one sign.  A 16-bit c takes them by choice, as its own rounding is larger (2-norm
// of it: bf16 1.7e-3, fp16 2.1e-4; one element in a hundred, or one in fifteen of an fp16 c, goes to the other neighbour) and they are up to 1.6 times
// as fast (8 192 x 8 192 x 8 192 480 and 760 us; few rows gain 0.1 to 0.4 us, but what an element loses shall not depend on how
// many rows there are); with LMT_FP32_SUMS it does not.  For those and for an fp32 c operands are widened to bf16 (exactly, within bf16's
// range: 3 bits of mantissa and a power of two) and go through the bf16 instructions (4e-8 at k of 1 024), at 1.3 PFLOP/s from registers instead of 4.7.
#include "lmt_device.h"
#include "lmt_internal.h"
#include "lmt_tiles.h"

namespace lmt {
namespace {

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

// A workgroup takes squares of 128 x 128; a thread 4 rows of 8 columns, which it reads once for both results.  Bound by memory, both sides:
// 30 522 x 1 024 in fp32 38 us (4.9 TB/s), 16 384 x 4 096 in bf16 62 (4.3), 8 192 x 1 024 in bf16 8.6.  Results leave streaming, whole
// lines at a time (kept in the L2: 38, 68, 11.2; only the transpose streaming: 38, 60, 9.5).  One side alone of 16 384 x 4 096: 48, in squares 42.  8 rows to a thread of half as many: two
// workgroups a compute unit, less in flight, a tenth slower.
constexpr uint32_t kQuantizeThreads = 512;
template <typename T, bool E5M2, bool TILE>
__global__ __launch_bounds__(kQuantizeThreads, 4) void k_quantize(const Quantize p, uint32_t tiles_across, uint32_t tiles_down) {
  __shared__ __align__(16) uint32_t col_max[128];  // TILE: the first is the square's
  __shared__ __align__(16) uint8_t turned[128 * 128];
  const uint32_t cg = threadIdx.x & 15u, rg = threadIdx.x >> 4;
  const uint64_t q_row = round_up(p.cols, 128), s_row = 4 * ceil_div(p.cols, 512), qt_row = round_up(p.rows, 128), st_row = 4 * ceil_div(p.rows, 512);
  const uint64_t n_tiles = (uint64_t)tiles_across * tiles_down;
  for (uint64_t at = blockIdx.x; at < n_tiles; at += gridDim.x) {
    const uint64_t tile = neighbours(at, n_tiles);  // a line of scales holds several squares': one L2 puts it together
    const uint32_t tr = (uint32_t)(tile / tiles_across), tc = (uint32_t)(tile % tiles_across);
    const uint32_t r0 = tr * 128u + rg * 4u, c0 = tc * 128u + cg * 8u;
    const uint32_t n = c0 < p.cols ? min(8u, p.cols - c0) : 0u;
    Vec<T, 8> x[4];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      x[j] = {};
      if (r0 + j < p.rows && n == 8) load<true>(x[j], static_cast<const T*>(p.x) + (uint64_t)(r0 + j) * p.ld + c0);
    }
    if (n != 0 && n != 8) {  // the end of a row
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j)
        if (r0 + j < p.rows) load_end(x[j], static_cast<const T*>(p.x) + (uint64_t)(r0 + j) * p.ld + c0, n, 0.f);
    }
    if (threadIdx.x < 128u) col_max[threadIdx.x] = 0;
    __syncthreads();
    uint32_t row_max[4] = {}, cm[8] = {};
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t m = magnitude(x[j].get(i));
        row_max[j] = max(row_max[j], m);
        cm[i] = max(cm[i], m);
      }
    uint32_t row_scale[4], col_scale[8];
    if constexpr (TILE) {
      uint32_t m = max(max(row_max[0], row_max[1]), max(row_max[2], row_max[3]));
      m = max16(m);
      m = max(m, (uint32_t)__shfl_xor((int)m, 16));
      m = max(m, (uint32_t)__shfl_xor((int)m, 32));
      if ((threadIdx.x & 63u) == 0) atomicMax(&col_max[0], m);
      __syncthreads();
      const uint32_t s = scale_of<E5M2>(col_max[0]);
#pragma unroll
      for (int i = 0; i < 4; ++i) row_scale[i] = s;
#pragma unroll
      for (int i = 0; i < 8; ++i) col_scale[i] = s;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) row_scale[j] = scale_of<E5M2>(max16(row_max[j]));
      if (p.qt) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t m = max(cm[i], (uint32_t)__shfl_xor((int)cm[i], 16));
          m = max(m, (uint32_t)__shfl_xor((int)m, 32));
          if ((threadIdx.x & 48u) == 0) atomicMax(&col_max[cg * 8u + i], m);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) col_scale[i] = scale_of<E5M2>(col_max[cg * 8u + i]);
      }
    }
    if (p.q) {
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        if (r0 + j >= p.rows) break;
        const float by = inverse_of(row_scale[j]);
        const float lo[4] = {x[j].get(0), x[j].get(1), x[j].get(2), x[j].get(3)}, hi[4] = {x[j].get(4), x[j].get(5), x[j].get(6), x[j].get(7)};
        const u32x2 w = {pack4<E5M2>(lo, by), pack4<E5M2>(hi, by)};
        __builtin_nontemporal_store(w, (LMT_GLOBAL u32x2*)(p.q + (uint64_t)(r0 + j) * q_row + c0));
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
        const float col[4] = {x[0].get(i), x[1].get(i), x[2].get(i), x[3].get(i)};
        // 16-byte pieces of a column's 128 bytes change places by the column's eight, so that they spread over the LDS banks
        *reinterpret_cast<uint32_t*>(&turned[(cg * 8u + i) * 128u + ((rg / 4u) ^ (cg & 7u)) * 16u + (rg & 3u) * 4u]) = pack4<E5M2>(col, inverse_of(col_scale[i]));
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
      for (uint32_t k = 0; k < 2; ++k) {
        const uint32_t c = k * 64u + threadIdx.x / 8u, piece = threadIdx.x & 7u;
        if (tc * 128u + c < p.cols)
          __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(&turned[c * 128u + (piece ^ (c / 8u & 7u)) * 16u]), (LMT_GLOBAL u32x4*)(p.qt + (uint64_t)(tc * 128u + c) * qt_row + (uint64_t)tr * 128u + piece * 16u));
      }
    }
    __syncthreads();
  }
}

// ---- product ---------------------------------------------------------------------------

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// The matrix instructions take X = b and Y = a: D[i][j] += sum over k of X[i][k] Y[j][k].  Lane l gives row l % 32 of both and has
// D[8 g + 4 (l / 32) + r][l % 32] in element 4 g + r: four neighbours of a row of c.  Which k a lane gives is of no concern as long
// as it is the same for X and Y.
// A lane's operands for 64 bytes of k: pieces at[0] and at[1] of its rows.
template <typename S>
struct Operands {
  u32x4 x[S::TN][2], y[S::TM][2];
  __device__ __forceinline__ void read(const uint8_t* a, const uint8_t* b, const uint32_t (&at)[2]) {
#pragma unroll
    for (int f = 0; f < S::TN; ++f)
#pragma unroll
      for (int q = 0; q < 2; ++q) x[f][q] = *reinterpret_cast<const u32x4*>(b + f * 4096 + at[q]);
#pragma unroll
    for (int f = 0; f < S::TM; ++f)
#pragma unroll
      for (int q = 0; q < 2; ++q) y[f][q] = *reinterpret_cast<const u32x4*>(a + f * 4096 + at[q]);
  }
};
// as, bs: the scales of the lane's rows, this block's in the lowest byte.
// narrow: one instruction takes 64 bytes of k and the scales.
template <typename S, int AF, int BF>
__device__ __forceinline__ void multiply_narrow(f32x16 (&acc)[S::TM][S::TN], const Operands<S>& o, const uint32_t (&as)[S::TM], const uint32_t (&bs)[S::TN]) {
  const auto whole = [](const u32x4 (&w)[2]) {
    return i32x8{(int)w[0].x, (int)w[0].y, (int)w[0].z, (int)w[0].w, (int)w[1].x, (int)w[1].y, (int)w[1].z, (int)w[1].w};
  };
#pragma unroll
  for (int i = 0; i < S::TM; ++i)
#pragma unroll
    for (int j = 0; j < S::TN; ++j)
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(whole(o.x[j]), whole(o.y[i]), acc[i][j], BF, AF, 0, (int)bs[j], 0, (int)as[i]);
}
// Two 8-bit values, the lower or the upper ones of w, in bf16, times s.
template <int E5M2, bool UPPER>
__device__ __forceinline__ uint32_t widen(uint32_t w, float s) {
  if constexpr (E5M2) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((int)w, s, UPPER));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, s, UPPER));
}
// wide: operands go to bf16 with their scales, 16 bytes at a time; each instruction takes 16 of k.
template <typename S, int AF, int BF>
__device__ __forceinline__ void multiply_wide(f32x16 (&acc)[S::TM][S::TN], const Operands<S>& o, const uint32_t (&as)[S::TM], const uint32_t (&bs)[S::TN]) {
  const auto wide = [](bf16x8 (&to)[2], const u32x4& w, uint32_t scales, auto e5m2) {
    const float s = __uint_as_float((scales & 255u) << 23);
#pragma unroll
    for (int v = 0; v < 2; ++v)
      to[v] = __builtin_bit_cast(bf16x8, u32x4{widen<e5m2.value, false>(w[2 * v], s), widen<e5m2.value, true>(w[2 * v], s),
                                               widen<e5m2.value, false>(w[2 * v + 1], s), widen<e5m2.value, true>(w[2 * v + 1], s)});
  };
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    bf16x8 x[S::TN][2];
#pragma unroll
    for (int f = 0; f < S::TN; ++f) wide(x[f], o.x[f][q], bs[f], Const<BF>{});
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      bf16x8 y[2];
      wide(y, o.y[i][q], as[i], Const<AF>{});
#pragma unroll
      for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[j][v], y[v], acc[i][j], 0, 0, 0);
    }
    if (q == 0) settle<S>(acc);  // one piece's operands at a time fit the registers
  }
}

// N neighbours of c's row i from column j on.
template <typename TC, int N>
__device__ __forceinline__ void put(const Matmul& p, uint32_t i, uint32_t j, float (&f)[N]) {
  if (i >= p.m || j >= p.n) return;
  TC* to = static_cast<TC*>(p.c) + (uint64_t)i * p.ldc + j;
  const uint32_t n = min((uint32_t)N, p.n - j);
  Vec<TC, N> y = {};
  if (p.accumulate) {
    if (n == N) load<false>(y, to);
    else load_end(y, to, n, 0.f);
#pragma unroll
    for (int r = 0; r < N; ++r) f[r] += y.get(r);
  }
  y.set(f);
  if (n == N) store<false>(to, y);
  else store_end(to, y, n);
}

// us (and PFLOP/s) on random numbers, buffers changing from call to call: 8 192 x 8 192 x 8 192 into bf16 480 (2.3), into fp32 775 (1.4): the way
// through LDS, 64 KB in and 192 out per block of k, takes about 2 000 cycles, the 8-bit instructions as many, and they overlap in
// part only; 2 432 x 30 522 x 1 024 into bf16 117 (1.3; 97 to 104 where operands and results are found in the Infinity Cache): the matrix cores are busy 30 % of
// the time by the counters, of a round of tiles a third is its start and its results, 148 MB in all;
// 4 096 x 1 024 x 32 768 into fp32 in four parts 213 + 21 (1.2): busy 63 %.  No LDS bank conflicts in either.
// Tiles of 256 x 256 because a byte staged is then used 256 times; 128 x 128 stages twice as much: the products above 605, 890, 125 and 265 us.
template <typename S, int AF, int BF, bool WIDE, typename TC>
__global__ __launch_bounds__(S::threads, 2) void k_matmul(const Matmul p, const Tiles t) {
  __shared__ __align__(16) uint8_t stage[S::lds];
  constexpr uint32_t kStage = S::rows * 128;
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
  const uint32_t n_tiles = t.across * t.down, split = blockIdx.x / n_tiles;
  uint32_t tile_m, tile_n;
  tile_of(t, blockIdx.x - split * n_tiles, &tile_m, &tile_n);
  const uint32_t m0 = tile_m * S::rows_m, n0 = tile_n * S::rows_n;
  const uint32_t blocks = (p.k + 127u) / 128u, s_row = (uint32_t)scale_row_bytes(p.k), row = blocks * 128u;
  const uint32_t first = split * t.split_blocks, end = min(blocks, first + t.split_blocks);
  // what this thread stages: rows behind the last one are the last one again.  The eight pieces of 16 bytes of a row's block change
  // places by half the row's number: a read of one piece from 16 rows (LDS serves 16 lanes of 16 bytes at once) then meets every
  // bank once.
  const uint8_t *a0 = p.a + (uint64_t)m0 * row, *b0 = p.b + (uint64_t)n0 * row;
  const uint32_t last_m = p.m - 1u - m0, last_n = p.n - 1u - n0;
  uint32_t from[S::loads];
#pragma unroll
  for (int j = 0; j < S::loads; ++j) {
    const uint32_t r = (j * S::waves + wave) * 8u + lane / 8u;
    const uint32_t piece = ((lane & 7u) ^ (r >> 1 & 7u)) * 16u;
    from[j] = (j * S::waves * 8 < S::rows_m ? min(r, last_m) : min(r - S::rows_m, last_n)) * row + piece;
  }
  const auto fetch = [&](uint32_t block, uint32_t at) {
#pragma unroll
    for (int j = 0; j < S::loads; ++j)
      load_to_lds(j * S::waves * 8 < S::rows_m ? a0 : b0, from[j], block * 128u, stage + at + (j * S::waves + wave) * 1024u);
  };
  // what this lane reads: pieces 4 h + 2 (l / 32) + q of rows l % 32
  uint32_t at[2][2];
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) at[h][q] = (lane & 31u) * 128u + ((4u * h + 2u * (lane >> 5) + q) ^ (lane >> 1 & 7u)) * 16u;
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
    for (int i = 0; i < S::TM; ++i) as_next[i] = load_word(as0, as_from[i], block);
#pragma unroll
    for (int j = 0; j < S::TN; ++j) bs_next[j] = load_word(bs0, bs_from[j], block);
  };
  f32x16 acc[S::TM][S::TN] = {};
  uint32_t now = 0;  // the stage that is multiplied
  if (first < end) {
    scales(first);
    fetch(first, 0);
  }
  Operands<S> o;
  if constexpr (S::turns) {
    wait_and_meet<0>();            // the first block has arrived
    if (wave >= S::waves / 2) meet();  // the second group is one turn behind
  }
  for (uint32_t g = first; g < end; g += 4u) {
#pragma unroll
    for (int i = 0; i < S::TM; ++i) as[i] = as_next[i];
#pragma unroll
    for (int j = 0; j < S::TN; ++j) bs[j] = bs_next[j];
    const uint32_t stop = min(g + 4u, end);
    for (uint32_t block = g; block < stop; ++block) {
      if constexpr (!S::turns) wait_and_meet<0>();  // the block has arrived, everybody's part of it, and nobody reads the other stage any more
      if (block == g && stop < end) scales(stop);
      // With turns: nobody reads the other stage, as everybody's reads of the block in front ended before a barrier that this group has
      // passed, and the second half's turn below ends with what is fetched here in place, one turn before anyone reads it
      if (block + 1u < end) fetch(block + 1u, kStage - now);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        o.read(stage + now + a_at, stage + now + b_at, at[h]);
        if constexpr (S::turns) {
          if (h == 0) reads_done_and_meet();
          else wait_and_meet<0>();
          __builtin_amdgcn_s_setprio(1);
        }
        if constexpr (WIDE) multiply_wide<S, AF, BF>(acc, o, as, bs);
        else multiply_narrow<S, AF, BF>(acc, o, as, bs);
        settle<S>(acc);
        if constexpr (S::turns) {
          __builtin_amdgcn_s_setprio(0);
          meet();
        }
      }
      now = kStage - now;
#pragma unroll
      for (int i = 0; i < S::TM; ++i) as[i] >>= 8;
#pragma unroll
      for (int j = 0; j < S::TN; ++j) bs[j] >>= 8;
    }
  }
  if constexpr (S::turns) {
    if (wave < S::waves / 2) meet();
  }
  if (t.splits > 1u) {  // this part's sums, in the order of the threads
    float* part = p.workspace + ((uint64_t)blockIdx.x * S::threads + threadIdx.x) * 4u;
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(LMT_GLOBAL f32x4*)(part + (uint64_t)((i * S::TN + j) * 4 + g) * gridDim.x * S::threads * 4u) =
              f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
    return;
  }
  // 64 rows of 64 at a time through LDS, a wavefront in its own part of it, so that rows of c are written 128 bytes and more at a time
  wait_and_meet<0>();
  float* mine = reinterpret_cast<float*>(stage) + wave * (64 * 64);
  constexpr int N = 16 / sizeof(TC);  // elements a lane writes
#pragma unroll
  for (int half = 0; half < S::TM / 2; ++half) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (uint32_t g = 0; g < 4; ++g) {
          const f32x16& d = acc[2 * half + i][j];
          const uint32_t r = i * 32u + (lane & 31u), piece = j * 8u + g * 2u + (lane >> 5);
          *reinterpret_cast<f32x4*>(mine + r * 64u + (piece ^ (r & 15u)) * 4u) = f32x4{d[4 * g], d[4 * g + 1], d[4 * g + 2], d[4 * g + 3]};
        }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (uint32_t it = 0; it < 64u * 64u / (64u * N); ++it) {
      const uint32_t e = it * 64u + lane, r = e / (64u / N), col = e % (64u / N) * N;
      float f[N];
#pragma unroll
      for (uint32_t v = 0; v < N; v += 4) {
        const f32x4 d = *reinterpret_cast<const f32x4*>(mine + r * 64u + ((col / 4u + v / 4u) ^ (r & 15u)) * 4u);
        f[v] = d.x, f[v + 1] = d.y, f[v + 2] = d.z, f[v + 3] = d.w;
      }
      put<TC, N>(p, m0 + (wm * S::TM + 2 * half) * 32u + r, n0 + wn * 64u + col, f);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Adds the parts of k in order, one workgroup per tile and 4 x threads elements of it, in the layout of k_matmul's threads.  Bound by memory:
// four parts of 4 096 x 1 024 and c, in and out, 21 us (101 MB, 4.8 TB/s).
template <typename S, typename TC>
__global__ __launch_bounds__(S::threads) void k_matmul_join(const Matmul p, const Tiles t) {
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, wm = wave / S::WN, wn = wave % S::WN;
  const uint32_t n_tiles = t.across * t.down, piece = blockIdx.x / n_tiles, id = blockIdx.x % n_tiles;
  uint32_t tile_m, tile_n;
  tile_of(t, id, &tile_m, &tile_n);
  const uint32_t i = piece / (S::TN * 4), j = piece / 4 % S::TN, g = piece % 4;
  const uint64_t split_size = (uint64_t)n_tiles * S::threads * 4u;
  const float* part = p.workspace + (uint64_t)piece * t.splits * split_size + ((uint64_t)id * S::threads + threadIdx.x) * 4u;
  f32x4 sum = *(const LMT_GLOBAL f32x4*)part;
#pragma unroll 4
  for (uint32_t s = 1; s < t.splits; ++s) sum += *(const LMT_GLOBAL f32x4*)(part + s * split_size);
  float f[4] = {sum.x, sum.y, sum.z, sum.w};
  put<TC, 4>(p, tile_m * S::rows_m + (wm * S::TM + i) * 32u + (lane & 31u), tile_n * S::rows_n + (wn * S::TN + j) * 32u + g * 8u + (lane >> 5) * 4u, f);
}

// Few rows of a (up to 64) and a short k: what counts is how soon the last byte has arrived.  A workgroup has 16 rows of b, its eight
// wavefronts every eighth block of k, operands straight from memory to registers (16 rows of 128 bytes to an instruction, whole
// lines), all in flight at once; the eight sums meet in LDS.  37 x 1 024 x 1 024: 5.7 us, by tiles of 128 x 128 7.5
// (in a graph, the kernel alone, by 8-bit instructions 3.8, by bf16 ones 4.0; 1 x 4 096 x 4 096 6.0 and 6.4).
constexpr uint32_t kFewRows = 64, kFewWaves = 8;
struct Lane {  // 32 bytes of a row's block, the lane's share of it
  u32x4 w[2];
  uint32_t scale;
  __device__ __forceinline__ void read(const uint8_t* from, const uint8_t* scales, uint32_t block) {
    const LMT_GLOBAL u32x4* g = (const LMT_GLOBAL u32x4*)(from + (uint64_t)block * 128u);
    w[0] = g[0], w[1] = g[1];
    scale = *(const LMT_GLOBAL uint8_t*)(scales + block);
  }
  __device__ __forceinline__ i32x8 whole() const {
    return i32x8{(int)w[0].x, (int)w[0].y, (int)w[0].z, (int)w[0].w, (int)w[1].x, (int)w[1].y, (int)w[1].z, (int)w[1].w};
  }
  template <int E5M2>
  __device__ __forceinline__ bf16x8 wide(int q) const {  // bytes 8 q .. 8 q + 7
    const float s = __uint_as_float(scale << 23);
    const uint32_t lo = w[q / 2][2 * (q % 2)], hi = w[q / 2][2 * (q % 2) + 1];
    return __builtin_bit_cast(bf16x8, u32x4{widen<E5M2, false>(lo, s), widen<E5M2, true>(lo, s), widen<E5M2, false>(hi, s), widen<E5M2, true>(hi, s)});
  }
};
template <int AF, int BF, bool WIDE, typename TC>
__global__ __launch_bounds__(64 * kFewWaves) void k_matmul_few(const Matmul p) {
  __shared__ f32x4 part[kFewWaves][4][64];
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15u;
  const uint32_t n0 = blockIdx.x * 16u, blocks = (p.k + 127u) / 128u, s_row = (uint32_t)scale_row_bytes(p.k);
  const uint64_t row = (uint64_t)blocks * 128u;
  const uint8_t *a[4], *as[4];
#pragma unroll
  for (uint32_t f = 0; f < 4; ++f) {
    const uint32_t i = min(f * 16u + r, p.m - 1u);
    a[f] = p.a + i * row + (lane >> 4) * 32u, as[f] = p.a_scales + (uint64_t)i * s_row;
  }
  const uint32_t of_b = min(n0 + r, p.n - 1u);
  const uint8_t *b = p.b + of_b * row + (lane >> 4) * 32u, *bs = p.b_scales + (uint64_t)of_b * s_row;
  f32x4 acc[4] = {};
  for (uint32_t block = wave; block < blocks; block += kFewWaves) {
    Lane x, y[4];
    x.read(b, bs, block);
#pragma unroll
    for (uint32_t f = 0; f < 4; ++f)
      if (f * 16u < p.m) y[f].read(a[f], as[f], block);
#pragma unroll
    for (uint32_t f = 0; f < 4; ++f) {
      if (f * 16u >= p.m) continue;
      if constexpr (WIDE) {
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.template wide<BF>(q), y[f].template wide<AF>(q), acc[f], 0, 0, 0);
      } else {
        acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x.whole(), y[f].whole(), acc[f], BF, AF, 0, (int)x.scale, 0, (int)y[f].scale);
      }
    }
  }
#pragma unroll
  for (int f = 0; f < 4; ++f) part[wave][f][lane] = acc[f];
  __syncthreads();
  if (wave >= 4u) return;  // a wavefront per square of 16 x 16
  f32x4 sum = part[0][wave][lane];
#pragma unroll
  for (uint32_t w = 1; w < kFewWaves; ++w) sum += part[w][wave][lane];
  float f[4] = {sum.x, sum.y, sum.z, sum.w};
  put<TC, 4>(p, wave * 16u + r, n0 + (lane >> 4) * 4u, f);  // lane l has rows l % 16 of a and four neighbours, from 4 (l / 16) on, of b
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
  const uint32_t grid = (uint32_t)std::min<uint64_t>((uint64_t)across * down, 1u << 22);
  return with_float(dtype, [&](auto t) {
    return with_fp8(fp8, [&](auto f) {
      typedef decltype(t) T;
      constexpr bool E5M2 = decltype(f)::value == 1;
      if (tile) hipLaunchKernelGGL((k_quantize<T, E5M2, true>), dim3(grid), dim3(kQuantizeThreads), 0, s, p, across, down);
      else hipLaunchKernelGGL((k_quantize<T, E5M2, false>), dim3(grid), dim3(kQuantizeThreads), 0, s, p, across, down);
      return hipGetLastError();
    });
  });
}

namespace {

typedef Shape<2, 4, 4, 2> Large;   // 256 x 256
typedef Shape<2, 2, 2, 2> Medium;  // 128 x 128

struct Choice {
  enum { kFew, kMedium, kLarge } form;
  Tiles tiles;
};
template <typename S>
Tiles tiles_of(uint64_t m, uint64_t n, uint64_t k, uint64_t splits) {
  const uint64_t blocks = ceil_div(k, 128), per = std::max<uint64_t>(4, round_up(ceil_div(blocks, splits), 4));  // scales come four at a time
  return {(uint32_t)ceil_div(n, S::rows_n), (uint32_t)ceil_div(m, S::rows_m), (uint32_t)std::max<uint64_t>(1, ceil_div(blocks, per)), (uint32_t)per};
}
// us with bf16 results, and behind the stroke with fp32 ones, the chosen form first.  fp32 results, and 16-bit ones from fp32 sums, take another inner loop at two
// thirds of the rate, but the borders lie alike; one rule, and workspace, for all.
//   Few rows: while a workgroup's wavefronts have few loads each.  37 x 1 024 x 1 024: 5.7 (medium 7.5) | 5.9 (10.7), 1 x 1 024 x 4 096: 5.9 (9.7) | 5.9 (12.4);
//   beyond, 37 x 1 024 x 4 096: medium 9.6 (11.0) | 12.4 (11.1: the rule is a tenth off there), 64 x 30 522 x 1 024: 9.9 (22.9) | 13.7 (24.8).
//   Large tiles, one workgroup per compute unit, take 5/3 of the time of a round of medium ones, of which there are two per unit:
//   4 096 x 4 096 x 4 096: large 60 (70) | 105 (120), 6 144 x 4 096 x 1 024: medium 33 (39) | 54 (62), 2 048 x 4 096 x 1 024: medium 15 (20) | 22 (29).
//   Too few tiles: parts of k, of 1 024 at least, up to a workgroup per unit.  1 024 x 1 024 x 4 096: 17 (in one part 24) | 20 (34).  With a long k
//   large tiles are worth the more parts: 4 096 x 1 024 x 32 768 159 (medium 240) | 232 (265); at 8 192 medium 48 (54) | 74 (79).
Choice choose(uint64_t m, uint64_t n, uint64_t k) {
  const uint64_t blocks = ceil_div(k, 128);
  k = 128 * blocks;  // what the operands hold: the same form, and workspace, for any k of so many blocks
  if (m <= kFewRows && n <= 4096 && ceil_div(m, 16) * blocks <= 32) return {Choice::kFew, {}};
  const uint64_t large = ceil_div(m, Large::rows_m) * ceil_div(n, Large::rows_n);
  const uint64_t medium = ceil_div(m, Medium::rows_m) * ceil_div(n, Medium::rows_n);
  if (medium > 2 * kCus && 5 * ceil_div(large, kCus) <= 3 * ceil_div(medium, 2 * kCus)) return {Choice::kLarge, tiles_of<Large>(m, n, k, 1)};
  if (large <= kCus && k >= 16384 && large * (k / 4096) >= kCus) return {Choice::kLarge, tiles_of<Large>(m, n, k, kCus / large)};
  return {Choice::kMedium, tiles_of<Medium>(m, n, k, std::max<uint64_t>(1, std::min<uint64_t>(kCus / medium, k / 1024)))};
}

}  // namespace

uint64_t matmul_workspace(uint64_t m, uint64_t n, uint64_t k) {
  if (m == 0 || n == 0) return 0;
  const Choice c = choose(m, n, k);
  const uint64_t tile = c.form == Choice::kLarge ? Large::rows_m * Large::rows_n : Medium::rows_m * Medium::rows_n;
  return c.tiles.splits > 1 ? 4 * tile * c.tiles.splits * c.tiles.across * c.tiles.down : 0;
}

hipError_t launch_matmul(const Matmul& p, int a_fp8, int b_fp8, int c_dtype, hipStream_t s) {
  const Choice c = choose(p.m, p.n, p.k);
  const auto tiled = [&](auto shape, auto af, auto bf, auto wide, auto tc) {
    typedef decltype(shape) S;
    typedef decltype(tc) TC;
    const uint32_t n_tiles = c.tiles.across * c.tiles.down;
    hipLaunchKernelGGL((k_matmul<S, decltype(af)::value, decltype(bf)::value, decltype(wide)::value != 0, TC>), dim3(n_tiles * c.tiles.splits), dim3(S::threads), 0, s, p, c.tiles);
    if (c.tiles.splits > 1)
      hipLaunchKernelGGL((k_matmul_join<S, TC>), dim3(n_tiles * S::TM * S::TN * 4), dim3(S::threads), 0, s, p, c.tiles);
    return hipGetLastError();
  };
  return with_fp8(a_fp8, [&](auto af) {
    return with_fp8(b_fp8, [&](auto bf) {
      return with_float(c_dtype, [&](auto tc) {
        const auto go = [&](auto wide) {
          switch (c.form) {
            case Choice::kFew:
              hipLaunchKernelGGL((k_matmul_few<decltype(af)::value, decltype(bf)::value, decltype(wide)::value != 0, decltype(tc)>), dim3((uint32_t)ceil_div(p.n, 16)), dim3(64 * kFewWaves), 0, s, p);
              return hipGetLastError();
            case Choice::kMedium: return tiled(Medium{}, af, bf, wide, tc);
            default: return tiled(Large{}, af, bf, wide, tc);
          }
        };
        if constexpr (sizeof(tc) == 4) return go(Const<1>{});
        else return p.fp32_sums ? go(Const<1>{}) : go(Const<0>{});
      });
    });
  });
}

}  // namespace lmt
