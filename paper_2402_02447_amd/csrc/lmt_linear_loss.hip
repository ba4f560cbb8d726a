// Cross entropy of x table^T without the logits, and the gradients of both (lmt.h).
//
// Logits are made twice.  The first time each tile leaves its rows' maxima and sums of exponentials, which are joined to a maximum and a sum a
// row; the second time, a piece of the classes at a time, tiles become g = w (softmax - onehot) in 16 bits, which is multiplied by the table (grad_x,
// summed over the pieces) and, as its columns, by x (grad_table).  Four products where three would do with the logits in memory; what is kept
// instead is one piece of g, of 2^27 elements at most, and the sums of grad_x, to which the pieces add one after the other.  g is rounded because the matrix instructions take both operands in one type (kFewRows).
#include "lmt_device.h"
#include "lmt_internal.h"
#include "lmt_tiles.h"

namespace lmt {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kInf = __builtin_inff();

__device__ __forceinline__ f32x16 mma(bf16_t, const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(_Float16, const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack2(bf16_t, float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2)); }
__device__ __forceinline__ uint32_t pack2(_Float16, float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, f16x2)); }
__device__ __forceinline__ float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32u) ? r[0] : r[1]);
}

// What the second pass knows of a row.  target: -1 for rows that are not counted.
struct RowOf {
  float top, log_sum, weight;  // log_sum: of the sum of exp(x - top), in units of log 2
  int target;
};

// ---- copies ---------------------------------------------------------------------------------

__device__ __forceinline__ int target_of(const void* targets, bool wide, uint64_t i, int64_t ignore, uint32_t classes, bool* bad) {
  const int64_t t = wide ? id_at<int64_t>(targets, i) : id_at<int32_t>(targets, i);
  *bad = t != ignore && (t < 0 || t >= (int64_t)classes);
  return t == ignore || *bad ? -1 : (int)t;
}
// A matrix with rows of whole blocks of 64, zeros behind their end: x and the table where they do not lie like that, and x with zeros in the rows that
// are not counted, for the table's gradient.  A thread 8 elements.  And what rows' targets and weights are.  One launch for all of it: 8 192 rows of 1 024 copied in 10 us.
struct Copy {
  const void* from;
  uint64_t ld;
  uint32_t rows, cols;
  bool counted;  // only the counted rows
  void* to;      // or nullptr
};
template <typename T>
__global__ __launch_bounds__(256) void k_linear_begin(const Copy a, const Copy b, const Copy c, const LinearLoss p, RowOf* rows, uint32_t* largest) {
  if (largest && blockIdx.x == 0 && threadIdx.x == 0) *largest = 0;
  for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < p.rows; i += gridDim.x * 256u) {
    bool bad;
    const int t = target_of(p.targets, p.wide_targets, i, p.ignore, p.classes, &bad);
    if (bad && p.status) atomicOr(p.status, LMT_STATUS_BAD_TARGET);
    rows[i] = {0.f, 0.f, t < 0 ? 0.f : p.weights ? load1(p.weights + i) : 1.f, t};
  }
  const uint32_t pieces = (uint32_t)(round_up(p.width, 64) / 8);
  for (int n = 0; n < 3; ++n) {
    const Copy& m = n == 0 ? a : n == 1 ? b : c;
    if (!m.to) continue;
    const uint64_t all = (uint64_t)m.rows * pieces;
    for (uint64_t of = (uint64_t)blockIdx.x * 256u + threadIdx.x; of < all; of += (uint64_t)gridDim.x * 256u) {
      const uint64_t i = of / pieces;
      const uint32_t j = (uint32_t)(of % pieces) * 8u;
      bool bad;
      Vec<T, 8> v;
      v.w[0] = v.w[1] = v.w[2] = v.w[3] = 0;
      if (j < m.cols && !(m.counted && target_of(p.targets, p.wide_targets, i, p.ignore, p.classes, &bad) < 0)) {
        const T* from = static_cast<const T*>(m.from) + i * m.ld + j;
        if (j + 8u <= m.cols) load<false>(v, from);
        else load_end(v, from, m.cols - j, 0.f);
      }
      *(LMT_GLOBAL u32x4*)(static_cast<T*>(m.to) + of * 8u) = u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
    }
  }
}

// ---- products -------------------------------------------------------------------------------

// c[i][j] = sum over k of a[i][k] b[j][k], or of operands that lie the other way, a[k][i] or b[k][j]: rows of whole blocks of 64 elements, 16-byte aligned.
struct Product {
  const uint8_t *a, *b;
  uint32_t a_row, b_row;  // bytes from row to row
  uint32_t m, n, k, blocks;  // k: rows of b where it lies the other way; a has whole blocks, zeros behind k
  Tiles t;
  uint32_t wrap;    // where a is twice as long, its rounding errors behind it: blocks of either part; b begins again there
  uint64_t a_more;  // bytes from one part of a to the other
  // what becomes of it
  const RowOf* rows;
  float2* sums;      // kStats: [tile of n][m]: maximum and sum of exp(x - maximum)
  float* hit;        // kStats: logit of the row's target
  // kGrad: [rows in whole blocks][g_ld], columns up to `cols`: g times its row's weight, and as it is, each with what rounding it leaves; or nullptr
  void *gw, *gw_left, *g, *g_left;
  uint64_t g_ld;
  uint32_t first_class, cols, classes;
  const uint32_t* largest;  // kGrad: bits of the largest weight
  void* c;           // kSum
  uint64_t ldc;
  bool accumulate, by_row;
  float* part;      // kSum: [split][m][n], sums that are joined later; `more`: added to those of the pieces in front
  bool more;
};
enum Mode { kStats, kGrad, kSum };

// bf16 has fp32's range: g has its row's weight in it, for both gradients.  In fp16 small weights would lose bits, so that there are two: without weights, times
// 2^14 (it is at most 1), for grad_x, whose rows get theirs at the end, and with them, times a power of two that brings the largest to 2^14, for grad_table.
// With few rows the products are small, and what rounding g leaves is kept and multiplied too: of both in fp16, where there are weights (76 rows, 2 003 classes,
// 257 columns 53 -> 56 us for the second pair).
template <typename T>
constexpr bool kNarrow = false;
template <>
constexpr bool kNarrow<_Float16> = true;
template <typename T>
constexpr float kRowScale = kNarrow<T> ? 0x1p14f : 1.f;
template <typename T>
__device__ __forceinline__ float column_scale(uint32_t largest) {
  if constexpr (!kNarrow<T>) return 1.f;
  const uint32_t e = max(largest >> 23, 1u);  // 2^(e - 127) <= largest < 2^(e - 126)
  return __uint_as_float(min(127u + 13u + 127u - min(e, 254u), 254u) << 23);
}

template <typename TC, int N>
__device__ __forceinline__ void put(TC* row, uint32_t j, uint32_t end, float (&f)[N], bool accumulate) {
  if (j >= end) return;
  TC* to = row + j;
  const uint32_t n = min((uint32_t)N, end - j);
  Vec<TC, N> y = {};
  if (accumulate) {
    if (n == N) load<false>(y, to);
    else load_end(y, to, n, 0.f);
#pragma unroll
    for (int r = 0; r < N; ++r) f[r] += y.get(r);
  }
  y.set(f);
  if (n == N) store<false>(to, y);
  else store_end(to, y, n);
}

// The loop is that of 8-bit products (one block of k arrives while another is multiplied, two groups of wavefronts in turns where there are
// eight), with 64 elements of 16 bits to a block.
// Operands that lie the other way (TURN_A, TURN_B) are staged as 64 rows of k, as many elements as the tile has rows, and read with the transposing
// read: 16 lanes read 4 rows of k of 16 elements, and get 4 k of an element each.  Their 64-byte parts change places by the row of k.
template <int ROWS>  // of the tile
struct Turned {
  static constexpr uint32_t pieces = ROWS / 8, row = ROWS * 2;
  // What thread `chunk` of a block's 16-byte pieces stages: row of k, and element.
  static __device__ __forceinline__ void place(uint32_t chunk, uint32_t* k, uint32_t* element) {
    *k = chunk / pieces, *element = (chunk % pieces ^ (*k & 3u) << 2) * 8u;
  }
  // Where a lane reads from for 32 elements from `first` on, k from 0 on.
  static __device__ __forceinline__ uint32_t at(uint32_t first, uint32_t lane) {
    const uint32_t k = 8u * (lane >> 5) + (lane >> 2 & 3u), element = first + 16u * (lane >> 4 & 1u) + 4u * (lane & 3u);
    return k * row + (element / 8u ^ (k & 3u) << 2) * 16u + (lane & 1u) * 8u;
  }
  // 16 k from 16 c on.
  static __device__ __forceinline__ u32x4 read(const uint8_t* from, int c) {
    typedef __attribute__((address_space(3))) s16x4* At;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(from + c * 16 * row)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(from + c * 16 * row + 4 * row)));
    return u32x4{lo.x, lo.y, hi.x, hi.y};
  }
};

// What bounds it is the turns of LDS and matrix cores, as with 8-bit products, and what a tile does before and behind its loop.  8 192 rows, 30 522 classes, 1 024 columns in bf16
// (512 GFLOP a product, in two pieces but for the statistics): statistics 455 us, 1.1 PFLOP/s; g 2 x 300, 0.85, 250 MB of it written each time; grad_x 2 x 222 and grad_table
// 2 x 225, 1.15, with one and two operands turned on the way from LDS.  (Copies of g and the table that lie along k instead, made by the kernels in front: 2 100 us in all for 1 910.)
template <typename S, typename T, Mode MODE, typename TC, bool TURN_A, bool TURN_B>
__global__ __launch_bounds__(S::threads, 2) void k_linear(const Product p) {
  __shared__ __align__(16) uint8_t stage[S::lds];
  __shared__ RowOf row_of[S::rows_m];
  constexpr uint32_t kStage = S::rows * 128;
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
  const uint32_t n_tiles = p.t.across * p.t.down, split = blockIdx.x / n_tiles;
  uint32_t tile_m, tile_n;
  tile_of(p.t, blockIdx.x - split * n_tiles, &tile_m, &tile_n);
  const uint32_t m0 = tile_m * S::rows_m, n0 = tile_n * S::rows_n;
  const uint32_t first = split * p.t.split_blocks, end = min(p.blocks, first + p.t.split_blocks);
  typedef Turned<S::rows_m> TurnedA;
  typedef Turned<S::rows_n> TurnedB;
  const uint8_t *a0 = p.a + (TURN_A ? 2ull * m0 : (uint64_t)m0 * p.a_row), *b0 = p.b + (TURN_B ? 2ull * n0 : (uint64_t)n0 * p.b_row);
  const uint32_t last_m = p.m - 1u - m0, last_n = p.n - 1u - n0;
  constexpr int kLoadsA = S::rows_m / (8 * S::waves);  // of 16 bytes per thread and block; the rest are b's
  uint32_t from[S::loads];
#pragma unroll
  for (int j = 0; j < S::loads; ++j) {
    const bool of_a = j < kLoadsA;
    if (of_a ? TURN_A : TURN_B) {
      uint32_t k, element;
      if (of_a) TurnedA::place((j * S::waves + wave) * 64u + lane, &k, &element), element = min(element, last_m & ~7u);
      else TurnedB::place(((j - kLoadsA) * S::waves + wave) * 64u + lane, &k, &element), element = min(element, last_n & ~7u);
      from[j] = k * (of_a ? p.a_row : p.b_row) + element * 2u;
    } else {
      const uint32_t r = (j * S::waves + wave) * 8u + lane / 8u;
      const uint32_t piece = ((lane & 7u) ^ (r >> 1 & 7u)) * 16u;
      from[j] = (of_a ? min(r, last_m) * p.a_row : min(r - S::rows_m, last_n) * p.b_row) + piece;
    }
  }
  const auto fetch = [&](uint32_t block, uint32_t at) {
    const uint32_t again = block >= p.wrap ? p.wrap : 0u, of_b = block - again;
    const uint8_t *a = a0 + (again ? p.a_more : 0ull) + (uint64_t)of_b * (TURN_A ? 64ull * p.a_row : 128ull), *b = b0 + (uint64_t)of_b * (TURN_B ? 64ull * p.b_row : 128ull);
    const bool end_b = TURN_B && of_b * 64u + 64u > p.k;  // b's rows of k behind the last one are the last one again, a has zeros there
#pragma unroll
    for (int j = 0; j < S::loads; ++j) {
      const bool of_a = j < kLoadsA;
      uint32_t offset = from[j];
      if (!of_a && end_b) {
        const uint32_t k = (((j - kLoadsA) * S::waves + wave) * 64u + lane) / TurnedB::pieces;
        offset -= (k - min(k, p.k - 1u - of_b * 64u)) * p.b_row;
      }
      send_to_lds(of_a ? a : b, offset, 0, stage + at + (j * S::waves + wave) * 1024u);
    }
  };
  uint32_t at[2][2], turned_a[S::TM], turned_b[S::TN];
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) at[h][q] = (lane & 31u) * 128u + ((4u * h + 2u * q + (lane >> 5)) ^ (lane >> 1 & 7u)) * 16u;
#pragma unroll
  for (uint32_t f = 0; f < S::TM; ++f) turned_a[f] = TurnedA::at((wm * S::TM + f) * 32u, lane);
#pragma unroll
  for (uint32_t f = 0; f < S::TN; ++f) turned_b[f] = S::rows_m * 128u + TurnedB::at((wn * S::TN + f) * 32u, lane);
  const uint32_t a_at = wm * S::TM * 4096u, b_at = S::rows_m * 128u + wn * S::TN * 4096u;
  if constexpr (MODE == kStats || MODE == kGrad) {
    if (threadIdx.x < S::rows_m) {
      RowOf r = {0.f, 0.f, 0.f, -1};
      if (m0 + threadIdx.x < p.m) r = p.rows[m0 + threadIdx.x];
      row_of[threadIdx.x] = r;
    }
  }
  f32x16 acc[S::TM][S::TN] = {};
  uint32_t now = 0;
  if (first < end) fetch(first, 0);
  u32x4 x[S::TN][2], y[S::TM][2];
  if constexpr (S::turns) {
    wait_and_meet<0>();
    if (wave >= S::waves / 2) meet();
  }
  for (uint32_t block = first; block < end; ++block) {
    if constexpr (!S::turns) wait_and_meet<0>();
    if (block + 1u < end) fetch(block + 1u, kStage - now);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int f = 0; f < S::TN; ++f)
#pragma unroll
        for (int q = 0; q < 2; ++q) x[f][q] = TURN_B ? TurnedB::read(stage + now + turned_b[f], 2 * h + q) : *reinterpret_cast<const u32x4*>(stage + now + b_at + f * 4096 + at[h][q]);
#pragma unroll
      for (int f = 0; f < S::TM; ++f)
#pragma unroll
        for (int q = 0; q < 2; ++q) y[f][q] = TURN_A ? TurnedA::read(stage + now + turned_a[f], 2 * h + q) : *reinterpret_cast<const u32x4*>(stage + now + a_at + f * 4096 + at[h][q]);
      if constexpr (S::turns) {
        if (h == 0) reads_done_and_meet();
        else wait_and_meet<0>();
        __builtin_amdgcn_s_setprio(1);
      }
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
          for (int j = 0; j < S::TN; ++j) acc[i][j] = mma(T{}, x[j][q], y[i][q], acc[i][j]);
      settle<S>(acc);
      if constexpr (S::turns) {
        __builtin_amdgcn_s_setprio(0);
        meet();
      }
    }
    now = kStage - now;
  }
  if constexpr (S::turns) {
    if (wave < S::waves / 2) meet();
  }
  wait_and_meet<0>();
  // lane l has row l % 32 of a's square, and of b's the rows 8 g + 4 (l / 32) + r in element 4 g + r
  if constexpr (MODE == kStats) {
    float2* part = reinterpret_cast<float2*>(stage);  // [wn][rows_m]
    const uint32_t c0 = n0 + wn * S::TN * 32u + 4u * (lane >> 5);
    const bool whole = n0 + S::rows_n <= p.n;
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      const uint32_t r = (wm * S::TM + i) * 32u + (lane & 31u);
      const int target = row_of[r].target;
      if (!whole) {
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[i][j][e] = c0 + 32u * j + 8u * (e / 4) + e % 4 < p.n ? acc[i][j][e] : -kInf;
      }
      float top = -kInf, sum = 0;
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, acc[i][j][e]);
      top = fmaxf(top, other_half(top));
      const float base = top == -kInf ? 0.f : top;
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f((acc[i][j][e] - base) * kLog2e);
      sum += other_half(sum);
      const uint32_t in = (uint32_t)target - c0;
      if (__builtin_amdgcn_ballot_w64(target >= 0 && in < 32u * S::TN) != 0) {
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (in == 32u * j + 8u * (e / 4) + e % 4 && target >= 0 && m0 + r < p.m) store1(p.hit + m0 + r, acc[i][j][e]);
      }
      if (lane < 32u) part[wn * S::rows_m + r] = {top, sum};
    }
    __syncthreads();
    if (threadIdx.x < S::rows_m && m0 + threadIdx.x < p.m) {
      float2 t[S::WN];
      float top = -kInf, sum = 0;
#pragma unroll
      for (int w = 0; w < S::WN; ++w) t[w] = part[w * S::rows_m + threadIdx.x], top = fmaxf(top, t[w].x);
#pragma unroll
      for (int w = 0; w < S::WN; ++w) sum += t[w].y == 0.f ? 0.f : t[w].y * __builtin_amdgcn_exp2f((t[w].x - top) * kLog2e);
      p.sums[(uint64_t)tile_n * p.m + m0 + threadIdx.x] = {top, sum};
    }
    return;
  }
  if constexpr (MODE == kGrad) {
    // 64 rows of 64 classes at a time through the wavefront's part of LDS, in 16 bits, so that they leave by whole lines; 16-byte pieces of a row change
    // places by its number
    uint8_t *places[2] = {stage + wave * 16384u, stage + wave * 16384u + 8192u};
    const float columns = column_scale<T>(load1(p.largest));
    const auto turn = [](uint32_t r) { return r >> 1 & 7u; };
    const auto left = [](uint32_t w, float a, float b) { return pack2(T{}, a - to_f32(__builtin_bit_cast(T, (uint16_t)w)), b - to_f32(__builtin_bit_cast(T, (uint16_t)(w >> 16)))); };
    const uint32_t c0 = n0 + wn * 64u, half = lane >> 5;
    const bool all_classes = p.first_class + c0 + 64u <= p.classes;
    // bf16: g times its weight, and what that leaves.  fp16: both, or with few rows one after the other, each with what it leaves.
    const bool few = p.gw_left || p.g_left;
#pragma unroll 1
    for (int pass = 0; pass < (kNarrow<T> && few ? 2 : 1); ++pass) {
      T* const to[2] = {static_cast<T*>(pass == 0 ? p.gw : p.g), static_cast<T*>(pass != 0 ? p.g_left : few ? p.gw_left : p.g)};
      if (!to[0] && !to[1]) continue;
#pragma unroll
      for (int two = 0; two < S::TM / 2; ++two) {
        const uint32_t r0 = (wm * S::TM + 2 * two) * 32u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t r = i * 32u + (lane & 31u);
          const RowOf of = row_of[r0 + r];
          const float by = pass == 0 ? of.weight * columns : kRowScale<T>;
          const uint32_t hit = (uint32_t)of.target - p.first_class - c0 - 4u * half;  // the target among this lane's classes
          const bool none = of.target < 0;
#pragma unroll
          for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (uint32_t g = 0; g < 4; ++g) {
              float f[4];
#pragma unroll
              for (uint32_t e = 0; e < 4; ++e) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[2 * two + i][j][4 * g + e] - of.top, kLog2e, -of.log_sum));
                f[e] = hit == 32u * j + 8u * g + e ? w - 1.f : w;
                if (!all_classes) f[e] = p.first_class + c0 + 4u * half + 32u * j + 8u * g + e < p.classes ? f[e] : 0.f;
              }
              const uint32_t at = r * 128u + ((j * 4u + g) ^ turn(r)) * 16u + half * 8u;
              const u32x2 v = none ? u32x2{0, 0} : u32x2{pack2(T{}, f[0] * by, f[1] * by), pack2(T{}, f[2] * by, f[3] * by)};
              *reinterpret_cast<u32x2*>(places[0] + at) = v;
              if (few) *reinterpret_cast<u32x2*>(places[1] + at) = none ? u32x2{0, 0} : u32x2{left(v.x, f[0] * by, f[1] * by), left(v.y, f[2] * by, f[3] * by)};
              else if (p.g) *reinterpret_cast<u32x2*>(places[1] + at) = none ? u32x2{0, 0} : u32x2{pack2(T{}, f[0] * kRowScale<T>, f[1] * kRowScale<T>), pack2(T{}, f[2] * kRowScale<T>, f[3] * kRowScale<T>)};
            }
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          if (!to[which]) continue;
#pragma unroll
          for (uint32_t it = 0; it < 8; ++it) {
            const uint32_t r = it * 8u + lane / 8u, piece = lane & 7u, i = m0 + r0 + r, j = c0 + piece * 8u;
            const u32x4 v = *reinterpret_cast<const u32x4*>(places[which] + r * 128u + (piece ^ turn(r)) * 16u);
            if (i < round_up(p.m, 64) && j < p.cols) *(LMT_GLOBAL u32x4*)(to[which] + (uint64_t)i * p.g_ld + j) = v;
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
    return;
  }
  // 64 rows of 64 at a time through LDS, a wavefront in its own part of it
  float* mine = reinterpret_cast<float*>(stage) + wave * (64 * 64);
  const float columns = p.largest ? 1.f / column_scale<T>(load1(p.largest)) : 1.f;
  float* part = p.part ? p.part + (uint64_t)split * p.m * p.n : nullptr;
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
    const uint32_t r0 = (wm * S::TM + 2 * half) * 32u, c0 = n0 + wn * 64u;
    constexpr int N = 16 / sizeof(TC);  // elements a lane writes
#pragma unroll
    for (uint32_t it = 0; it < 64u * 64u / (64u * N); ++it) {
      const uint32_t e = it * 64u + lane, r = e / (64u / N), col = e % (64u / N) * N;
      float f[N];
#pragma unroll
      for (uint32_t v = 0; v < N; v += 4) {
        const f32x4 d = *reinterpret_cast<const f32x4*>(mine + r * 64u + ((col / 4u + v / 4u) ^ (r & 15u)) * 4u);
        f[v] = d.x, f[v + 1] = d.y, f[v + 2] = d.z, f[v + 3] = d.w;
      }
      const uint32_t i = m0 + r0 + r, j = c0 + col;
      if (i >= p.m) continue;
      if (part) {
        put<float, N>(part + (uint64_t)i * p.n, j, p.n, f, p.more);
      } else {
        const float by = p.by_row ? p.rows[i].weight * (1.f / kRowScale<T>) : columns;
        const bool none = p.by_row && p.rows[i].target < 0;
#pragma unroll
        for (int v = 0; v < N; ++v) f[v] = none ? 0.f : f[v] * by;
        put<TC, N>(static_cast<TC*>(p.c) + (uint64_t)i * p.ldc, j, p.n, f, p.accumulate);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Adds the parts of a product in order, a thread 4 neighbours.  Memory: two parts of 8 192 x 1 024 in 14 us, 6 TB/s.
template <typename T, typename TC>
__global__ __launch_bounds__(256) void k_linear_join(const Product p, uint32_t parts) {
  const uint64_t across = ceil_div(p.n, 4), n = (uint64_t)p.m * across;
  for (uint64_t of = (uint64_t)blockIdx.x * 256u + threadIdx.x; of < n; of += (uint64_t)gridDim.x * 256u) {
    const uint64_t i = of / across;
    const uint32_t j = (uint32_t)(of % across) * 4u, left = min(4u, p.n - j);
    float f[4] = {};
    for (uint32_t part = 0; part < parts; ++part) {
      const float* from = p.part + ((uint64_t)part * p.m + i) * p.n + j;
      Vec<float, 4> v;
      if (left == 4u) load<false>(v, from);
      else load_end(v, from, left, 0.f);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] += v.get(e);
    }
    const float by = p.by_row ? p.rows[i].weight * (1.f / kRowScale<T>) : p.largest ? 1.f / column_scale<T>(load1(p.largest)) : 1.f;
    const bool none = p.by_row && p.rows[i].target < 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = none ? 0.f : f[e] * by;
    put<TC, 4>(static_cast<TC*>(p.c) + i * p.ldc, j, p.n, f, p.accumulate);
  }
}

// ---- rows ---------------------------------------------------------------------------------------

// Behind the first pass: the tiles' maxima and sums joined, the loss.  16 threads a row, each an equal part of the tiles, then one after the other, in order.  8 192 rows, 120 tiles: 12 us.
__device__ __forceinline__ float2 joined(float2 a, float2 b) {
  const float top = fmaxf(a.x, b.x);
  return {top, (a.y == 0.f ? 0.f : a.y * __builtin_amdgcn_exp2f((a.x - top) * kLog2e)) + (b.y == 0.f ? 0.f : b.y * __builtin_amdgcn_exp2f((b.x - top) * kLog2e))};
}
__global__ __launch_bounds__(256) void k_linear_rows(const LinearLoss p, RowOf* rows, const float2* sums, const float* hit, uint32_t tiles, uint32_t* largest) {
  __shared__ float2 part[16][17];
  const uint32_t of = threadIdx.x / 16u, row = threadIdx.x % 16u, i = blockIdx.x * 16u + row, each = (tiles + 15u) / 16u;
  float2 x = {-kInf, 0.f};
  if (i < p.rows)
    for (uint32_t t = of * each; t < min(tiles, (of + 1u) * each); ++t) x = joined(x, sums[(uint64_t)t * p.rows + i]);
  part[of][row] = x;
  __syncthreads();
  if (threadIdx.x >= 16u) return;
#pragma unroll
  for (uint32_t t = 1; t < 16; ++t) x = joined(x, part[t][row]);
  if (i >= p.rows) return;
  RowOf r = rows[i];
  const float log_sum = __builtin_amdgcn_logf(x.y);
  if (p.lse) store1(p.lse + i, __builtin_fmaf(log_sum, kLn2, x.x));
  if (p.loss) store1(p.loss + i, r.target < 0 ? 0.f : r.weight * __builtin_fmaf(log_sum, kLn2, x.x - load1(hit + i)));
  r.top = x.x, r.log_sum = log_sum;
  rows[i] = r;
  const uint32_t size = __float_as_uint(r.weight) & 0x7fffffffu;
  if (largest && size < 0x7f800000u) atomicMax(largest, size);
}

// ---- host ---------------------------------------------------------------------------------------

typedef Shape<2, 4, 4, 2> Large;   // 256 x 256
typedef Shape<2, 2, 2, 2> Medium;  // 128 x 128

struct Choice {
  bool large;
  Tiles t;
};
// What a form takes, in thirds of a microsecond: a round of large tiles, one a compute unit, 5 a block of k, one of medium ones, two a unit, 3; parts of k
// where `split`, each written and read once in fp32 at 5 TB/s.  (Four stages instead of two for few medium tiles: 76 x 2 003 x 257 10.4 us and 11.9.)
Choice choose(uint64_t m, uint64_t n, uint64_t blocks, bool split) {
  Choice best = {};
  double least = 0;
  for (const bool wide : {true, false}) {
    const uint64_t tile = wide ? 256 : 128, across = ceil_div(n, tile), down = ceil_div(m, tile), slots = wide ? kCus : 2 * kCus;
    for (uint64_t splits = 1; splits <= (split ? 16 : 1); ++splits) {
      const uint64_t per = std::max<uint64_t>(1, ceil_div(blocks, splits));
      if (splits > 1 && (per < 8 || ceil_div(blocks, per) != splits)) continue;
      const double takes = (double)ceil_div(across * down * splits, slots) * (double)(per + 4) * (wide ? 5 : 3) + (splits > 1 ? (double)(splits * m * n) * 8 / 5e6 * 3 + 12 : 0);
      if (least == 0 || takes < least) least = takes, best = {wide, {(uint32_t)across, (uint32_t)down, (uint32_t)splits, (uint32_t)per}};
    }
  }
  return best;
}

// Where things lie in the workspace, in bytes.
struct Plan {
  uint64_t piece, pieces;             // classes of a piece, a multiple of 256
  uint64_t parts, g_bytes;            // of g: 2 with what rounding leaves, one behind the other; each has so many bytes
  uint64_t x_row;                     // elements of padded rows of x and the table
  Choice stats, grad_x, grad_t;
  uint64_t rows, sums, hit, largest, x, table, counted, g, gw, part_x, part_t, end;
};
// Up to which what rounding g leaves is multiplied too.  A rule of cost alone: the products are twice as long.  That rounding is 1.7e-3 of a bf16 gradient's 2-norm at any
// number of rows (nearly all of it that of a weight times a target's element; the gradient's own rounding is as much again).
constexpr uint64_t kFewRows = 256;
constexpr uint64_t kPiece = 1ull << 27;  // elements of g at a time: 256 MB (in half of that 2 432 rows of 30 522 classes and 1 024 columns take 708 us for 654)
Plan plan_of(uint64_t n, uint64_t classes, uint64_t width, bool gradients, bool narrow, bool x_copy, bool table_copy) {
  Plan w = {};
  w.x_row = round_up(width, 64);
  w.parts = n <= kFewRows ? 2 : 1;
  w.pieces = std::max<uint64_t>(1, ceil_div(n * classes, kPiece));
  w.piece = std::min(round_up(ceil_div(classes, w.pieces), 256), round_up(classes, 256));
  w.pieces = ceil_div(classes, w.piece);
  w.stats = choose(n, classes, w.x_row / 64, false);
  w.grad_x = choose(n, width, w.parts * w.piece / 64, true);
  w.grad_t = choose(w.piece, width, w.parts * ceil_div(n, 64), true);
  const auto take = [&](uint64_t bytes) {
    const uint64_t at = w.end;
    w.end += round_up(bytes, 256);
    return at;
  };
  w.rows = take(n * sizeof(RowOf)), w.sums = take(w.stats.t.across * n * sizeof(float2)), w.hit = take(n * 4), w.largest = take(4);
  w.x = x_copy ? take(n * w.x_row * 2) : 0, w.table = table_copy ? take(classes * w.x_row * 2) : 0;
  if (gradients) {
    w.counted = take(n * w.x_row * 2);
    w.g_bytes = round_up(n, 64) * w.piece * 2;
    w.gw = take(w.parts * w.g_bytes), w.g = narrow ? take(w.parts * w.g_bytes) : 0;
    if (w.pieces > 1 || w.grad_x.t.splits > 1) w.part_x = take(w.grad_x.t.splits * n * width * 4);
    if (w.grad_t.t.splits > 1) w.part_t = take(w.grad_t.t.splits * w.piece * width * 4);
  }
  return w;
}

template <typename T, Mode MODE, typename TC, bool TURN_A, bool TURN_B>
void launch(Product p, Choice c, hipStream_t s) {
  if (p.wrap == 0) p.wrap = ~0u;
  const uint32_t grid = p.t.across * p.t.down * p.t.splits;
  if (c.large) hipLaunchKernelGGL((k_linear<Large, T, MODE, TC, TURN_A, TURN_B>), dim3(grid), dim3(Large::threads), 0, s, p);
  else hipLaunchKernelGGL((k_linear<Medium, T, MODE, TC, TURN_A, TURN_B>), dim3(grid), dim3(Medium::threads), 0, s, p);
}
template <typename T, typename TC>
void join(const Product& p, uint32_t parts, hipStream_t s) {
  hipLaunchKernelGGL((k_linear_join<T, TC>), dim3((uint32_t)std::min<uint64_t>(ceil_div((uint64_t)p.m * ceil_div(p.n, 4), 256), 1u << 16)), dim3(256), 0, s, p, parts);
}

// Whether rows can be read as they lie: on 16 bytes, of whole blocks.
bool as_it_is(const LinearLoss& q, const void* x, uint64_t ld) { return q.width % 64 == 0 && ld % 8 == 0 && ((uintptr_t)x & 15u) == 0 && ld <= LMT_MAX_WIDTH; }
Plan plan_of(const LinearLoss& q, bool narrow) {
  return plan_of(q.rows, q.classes, q.width, q.grad_x || q.grad_table, narrow, !as_it_is(q, q.x, q.x_ld), !as_it_is(q, q.table, q.table_ld));
}

template <typename T>
hipError_t launch_typed(const LinearLoss& q, hipStream_t s) {
  const bool gradients = q.grad_x || q.grad_table;
  const Plan w = plan_of(q, kNarrow<T>);
  uint8_t* base = static_cast<uint8_t*>(q.workspace);
  const auto at = [&](uint64_t offset) { return base + offset; };
  RowOf* rows = reinterpret_cast<RowOf*>(at(w.rows));
  uint32_t* largest = gradients ? reinterpret_cast<uint32_t*>(at(w.largest)) : nullptr;
  const bool x_copy = !as_it_is(q, q.x, q.x_ld), table_copy = !as_it_is(q, q.table, q.table_ld);
  const Copy x{q.x, q.x_ld, q.rows, q.width, false, x_copy ? at(w.x) : nullptr}, table{q.table, q.table_ld, q.classes, q.width, false, table_copy ? at(w.table) : nullptr};
  const Copy counted{q.x, q.x_ld, q.rows, q.width, true, q.grad_table ? at(w.counted) : nullptr};
  const uint64_t most = std::max<uint64_t>({x_copy || q.grad_table ? (uint64_t)q.rows * w.x_row : 0, table_copy ? (uint64_t)q.classes * w.x_row : 0, 8ull * q.rows});
  hipLaunchKernelGGL((k_linear_begin<T>), dim3((uint32_t)std::min<uint64_t>(ceil_div(most, 2048), 1u << 16)), dim3(256), 0, s, x, table, counted, q, rows, largest);
  Product p = {};
  p.a = x_copy ? at(w.x) : static_cast<const uint8_t*>(q.x), p.a_row = (uint32_t)(2 * (x_copy ? w.x_row : q.x_ld));
  p.b = table_copy ? at(w.table) : static_cast<const uint8_t*>(q.table), p.b_row = (uint32_t)(2 * (table_copy ? w.x_row : q.table_ld));
  p.m = q.rows, p.n = q.classes, p.blocks = (uint32_t)(w.x_row / 64), p.t = w.stats.t, p.rows = rows;
  p.sums = reinterpret_cast<float2*>(at(w.sums)), p.hit = reinterpret_cast<float*>(at(w.hit));
  p.classes = q.classes, p.largest = largest;
  launch<T, kStats, float, false, false>(p, w.stats, s);
  hipLaunchKernelGGL(k_linear_rows, dim3((uint32_t)ceil_div(q.rows, 16)), dim3(256), 0, s, q, rows, p.sums, p.hit, w.stats.t.across, largest);
  for (uint64_t piece = 0; gradients && piece < w.pieces; ++piece) {
    const uint32_t first = (uint32_t)(piece * w.piece), n = (uint32_t)std::min<uint64_t>(w.piece, q.classes - first);
    Product g = p;
    g.b = p.b + (uint64_t)first * p.b_row, g.n = n, g.first_class = first, g.cols = (uint32_t)round_up(n, 64), g.g_ld = w.piece;
    const Choice c = choose(q.rows, n, p.blocks, false);
    const bool unweighted = kNarrow<T> && (q.weights || w.parts == 1);  // grad_x from g without weights
    const auto made = [&](bool wanted, uint64_t place, void** whole, void** left) { *whole = wanted ? at(place) : nullptr, *left = wanted && w.parts > 1 ? at(place + w.g_bytes) : nullptr; };
    g.t = c.t, made(q.grad_table || !unweighted, w.gw, &g.gw, &g.gw_left), made(unweighted && q.grad_x, w.g, &g.g, &g.g_left);
    launch<T, kGrad, T, false, false>(g, c, s);
    if (q.grad_x) {  // g by the table's rows
      Product d = {};
      d.a = at(unweighted ? w.g : w.gw), d.a_row = (uint32_t)(2 * w.piece), d.b = g.b, d.b_row = p.b_row;
      d.m = q.rows, d.n = q.width, d.k = n, d.blocks = (uint32_t)w.parts * g.cols / 64, d.wrap = g.cols / 64, d.a_more = w.g_bytes, d.t = w.grad_x.t, d.rows = rows, d.by_row = unweighted, d.largest = unweighted ? nullptr : largest;
      d.c = q.grad_x, d.ldc = q.grad_x_ld;
      if (w.pieces > 1 || d.t.splits > 1) d.part = reinterpret_cast<float*>(at(w.part_x)), d.more = piece > 0;
      launch<T, kSum, T, false, true>(d, w.grad_x, s);
      if (d.part && piece + 1 == w.pieces) join<T, T>(d, d.t.splits, s);
    }
    if (q.grad_table) {  // g's columns by x's
      const auto typed = [&](auto tc) {
        typedef decltype(tc) TC;
        Product d = {};
        d.a = at(w.gw), d.a_row = (uint32_t)(2 * w.piece), d.b = at(w.counted), d.b_row = (uint32_t)(2 * w.x_row);
        d.m = n, d.n = q.width, d.k = q.rows, d.wrap = (uint32_t)ceil_div(q.rows, 64), d.blocks = (uint32_t)w.parts * d.wrap, d.a_more = w.g_bytes, d.largest = largest, d.accumulate = q.accumulate;
        d.t = w.grad_t.t, d.t.down = (uint32_t)ceil_div(n, w.grad_t.large ? Large::rows_m : Medium::rows_m);
        d.c = static_cast<TC*>(q.grad_table) + (uint64_t)first * q.grad_table_ld, d.ldc = q.grad_table_ld;
        if (d.t.splits > 1) d.part = reinterpret_cast<float*>(at(w.part_t));
        launch<T, kSum, TC, true, true>(d, w.grad_t, s);
        if (d.t.splits > 1) join<T, TC>(d, d.t.splits, s);
      };
      if (q.grad_table_f32) typed(float{});
      else typed(T{});
    }
  }
  return hipGetLastError();
}

}  // namespace

uint64_t linear_loss_workspace(uint64_t rows, uint64_t classes, uint64_t width, bool gradients) {
  return rows && classes ? std::max(plan_of(rows, classes, width, gradients, false, true, true).end, plan_of(rows, classes, width, gradients, true, true, true).end) : 0;
}
uint64_t linear_loss_workspace_of(int dtype, uint64_t rows, uint64_t classes, uint64_t width, bool gradients) {
  return rows && classes ? plan_of(rows, classes, width, gradients, dtype == LMT_F16, width % 64 != 0, width % 64 != 0).end : 0;
}
uint64_t linear_loss_workspace(const LinearLoss& p, int dtype) { return plan_of(p, dtype == LMT_F16).end; }
hipError_t launch_linear_loss(const LinearLoss& p, int dtype, hipStream_t s) {
  return dtype == LMT_F16 ? launch_typed<_Float16>(p, s) : launch_typed<bf16_t>(p, s);
}

}  // namespace lmt
