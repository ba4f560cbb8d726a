// Attention within the sequences of a packed batch, and its gradient (lmt.h).
//
// Which rows a row sees is an interval: its sequence, cut at the row itself where it is causal, no further down than the prefix.  The same
// holds for the rows that see a key.  So every mask is two numbers a row, a workgroup takes a block of rows whatever sequences they are of,
// and the keys it goes over are those from the first to the last that one of its rows sees; blocks of 32 x 32 inside all rows' intervals are
// not masked at all, those outside of a wavefront's rows not computed.
//
// One pass over the keys: with m a running maximum of the scores (in units of log 2), l = sum 2^(s - m) and o = sum 2^(s - m) v; when
// a score exceeds m by more than 2^kSlack both are multiplied by 2^(m - m') first.
//
// Matrix instructions (32 x 32 x 16, fp32 sums): lane l gives row l % 32 of both operands, eight k from 8 (l / 32) on, and has column
// l % 32 of the result, rows 8 g + 4 (l / 32) + r in element 4 g + r.  Scores are made as K Q^T, so that a lane has those of one query;
// what it has of them after exp2 is, in its order, an operand of V^T P^T again: no lane needs another one's.  V^T comes from
// LDS through the transposing read: 16 lanes read 4 rows of 16 elements, and get 4 rows' elements of a column each.
//
// Weights and derivatives are rounded to the type of what they multiply, since the instructions take both operands in one: half a step of theirs each, so that results are off by 1.2 to
// 1.45 times what rounding them alone is (bf16, in the 2-norm: 2.0e-3 for 1.6e-3, gradients 2.4e-3 for 1.8e-3).  In two pieces they would lose nothing and take those products twice.
#include <utility>

#include "lmt_device.h"
#include "lmt_internal.h"
#include "lmt_tiles.h"

namespace lmt {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#define LMT_LDS __attribute__((address_space(3)))

constexpr int kWaves = 4, kRows = 32 * kWaves, kThreads = 64 * kWaves;  // a wavefront has 32 rows
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ f32x16 mma(bf16_t, const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(_Float16, const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack2(bf16_t, float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2)); }
__device__ __forceinline__ uint32_t pack2(_Float16, float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, f16x2)); }

// f(0), f(1), ... f(N - 1), each with a number that is known when it is compiled: registers are not indexed.
template <typename F, int... I>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  each_of(std::make_integer_sequence<int, N>{}, f);
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
// A lane's value and that of the lane 32 further or back, joined.
__device__ __forceinline__ float halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ bool any(bool x) { return __builtin_amdgcn_ballot_w64(x) != 0; }
// The largest of the lanes up to this one, by moves between lanes: within rows of 16, then from the end of the rows in front.  -1 is the least.
__device__ __forceinline__ int max_so_far(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(-1, x, 0x111, 0xf, 0xf, false));  // row_shr:1
  x = max(x, __builtin_amdgcn_update_dpp(-1, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(-1, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(-1, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(-1, x, 0x142, 0xa, 0xf, false));  // row_bcast:15, to the second and fourth row
  return max(x, __builtin_amdgcn_update_dpp(-1, x, 0x143, 0xc, 0xf, false));  // row_bcast:31, to the upper half
}
// The largest and smallest of a wavefront's whole numbers of 0 and more.
__device__ __forceinline__ int wave_max(int x) { return __builtin_amdgcn_readlane(max_so_far(x), 63); }
__device__ __forceinline__ int wave_min(int x) { return 0x7fffffff - wave_max(0x7fffffff - x); }
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
  return x;
}

// ---- who sees whom -----------------------------------------------------------------------

// Of kRows rows in a row: the interval of what each sees (or, of keys: of who sees it), [lo, hi), 0 and 0 for nothing, -1 and -1 for rows that are another
// workgroup's or none; and where all of them lie.
struct Seen {
  int lo[kRows], hi[kRows], first, last, sequence;
};

// The sequence of a row is the last one that starts at or before it.
struct Sequence {
  int start, stop, prefix;
  __device__ __forceinline__ void read(const Attention& p, int s) {
    const int rows = (int)p.rows;
    start = min(max(load1(p.starts + s), 0), rows);
    int length = max(min(load1(p.starts + s + 1), rows) - start, 0);
    if (p.lengths) length = min(length, max(load1(p.lengths + s), 0));
    stop = start + length, prefix = p.causal && p.prefixes ? start + min(max(load1(p.prefixes + s), 0), length) : start;
  }
  template <bool KEYS>
  __device__ __forceinline__ void seen(const Attention& p, int i, int* lo, int* hi) const {
    if constexpr (KEYS) *lo = p.causal && i >= prefix ? i : start, *hi = stop;
    else *lo = start, *hi = p.causal ? max(i + 1, prefix) : stop;
  }
};

// A workgroup's rows: a block of kRows, or, where blocks are cut at the starts of sequences (p.cuts of them, so that a block that has rows of two long ones
// does not go over both), what a sequence that starts inside a block has of it.
struct Block {
  int first;  // row
  int cut;    // the sequence, or -1
  __device__ __forceinline__ void set(const Attention& p, uint32_t tile) {
    cut = tile < p.cuts ? (int)tile : -1;
    first = cut >= 0 ? min(max(load1(p.starts + cut), 0), (int)p.rows) : (int)((tile - p.cuts) * kRows);
  }
};

// Sequences that start in the block mark their first row, one more pass takes the running maximum; with many sequences the range that can
// matter is narrowed by a sample of them first.
template <bool KEYS>
__device__ __forceinline__ void find_seen(const Attention& p, const Block& block, Seen& s) {
  static_assert(kRows == 128 && kRows <= kThreads, "a thread a row, two wavefronts of them");
  const int t = (int)threadIdx.x, r0 = block.first, r1 = r0 + kRows, rows = (int)p.rows;
  const LMT_GLOBAL int32_t* starts = (const LMT_GLOBAL int32_t*)p.starts;
  if (t < kRows) s.lo[t] = -1;
  if (t == 0) s.first = 0x7fffffff, s.last = 0;
  __syncthreads();
  int of = -1;
  if (block.cut < 0) {
    uint32_t begin = 0, end = p.sequences;
    while (end - begin > 2u * kThreads) {
      const uint32_t step = (end - begin + kThreads - 1u) / kThreads, at = begin + (uint32_t)t * step;
      const int start = at < end ? starts[at] : 0x7fffffff;
      const uint32_t below = (uint32_t)__syncthreads_count(start <= r0), inside = (uint32_t)__syncthreads_count(start < r1);
      const uint32_t b = begin + (below ? below - 1u : 0u) * step, e = min(end, begin + inside * step);
      if (e <= b || e - b >= end - begin) {
        if (e <= b) end = begin;
        break;
      }
      begin = b, end = e;
    }
    for (uint32_t q = begin + (uint32_t)t; q < end; q += kThreads) {
      const int start = starts[q];
      if (start < r1) atomicMax(&s.lo[start <= r0 ? 0 : start - r0], (int)q);
    }
    __syncthreads();
    if (t < kRows) {
      of = max_so_far(s.lo[t]);
      if (t >= 64) of = max(of, wave_max(s.lo[t - 64]));
    }
    if (t == 0) s.sequence = of;
    __syncthreads();
  }
  if (t < kRows) {
    const int i = r0 + t;
    int lo = -1, hi = -1;
    Sequence sequence;
    if (block.cut >= 0) {
      sequence.read(p, block.cut);
      const int end = r0 % kRows ? min(sequence.stop, r0 / kRows * kRows + kRows) : 0;  // one that starts with a block has it all
      if (i < end) sequence.seen<KEYS>(p, i, &lo, &hi);
    } else if (i < rows) {
      lo = hi = 0;
      if (of >= 0) {
        sequence.read(p, of);
        if (i < sequence.stop) {
          if (p.cuts && of != s.sequence) lo = hi = -1;
          else sequence.seen<KEYS>(p, i, &lo, &hi);
        }
      }
    }
    s.lo[t] = lo, s.hi[t] = hi;
    const int first = wave_min(lo < hi ? lo : 0x7fffffff), last = wave_max(hi);
    if ((t & 63) == 0) atomicMin(&s.first, first), atomicMax(&s.last, last);
  }
  __syncthreads();
}

// One workgroup of a call looks the table over.
__device__ __forceinline__ void check_sequences(const Attention& p) {
  if (!p.status || blockIdx.x != 0) return;
  const LMT_GLOBAL int32_t* starts = (const LMT_GLOBAL int32_t*)p.starts;
  const int rows = (int)p.rows;
  bool bad = false;
  for (uint32_t s = threadIdx.x; s < p.sequences; s += blockDim.x) {
    const int a = starts[s], b = starts[s + 1u];
    bad |= a < 0 || b < a || b > rows;
    if (p.lengths) {
      const int n = ((const LMT_GLOBAL int32_t*)p.lengths)[s];
      bad |= n < 0 || (int64_t)a + n > b;
    }
  }
  if (bad) atomicOr(p.status, LMT_STATUS_BAD_SEQUENCE);
}

// A lane's row among what its wavefront and block see.
struct Span {
  int lo, hi;                              // of the lane's row
  int any_lo, any_hi, all_lo, all_hi;      // what some row of the wavefront sees, what all that see anything do
  __device__ __forceinline__ void read(const Seen& s, uint32_t row) {
    lo = s.lo[row], hi = s.hi[row];
    const bool some = lo < hi;
    any_lo = wave_min(some ? lo : 0x7fffffff), any_hi = wave_max(hi);
    all_lo = wave_max(lo), all_hi = wave_min(some ? hi : 0x7fffffff);
  }
  __device__ __forceinline__ bool mine() const { return hi >= 0; }
  __device__ __forceinline__ bool some() const { return lo < hi; }
  __device__ __forceinline__ bool touches(int at, int n) const { return at < any_hi && at + n > any_lo; }
  __device__ __forceinline__ bool inside(int at, int n) const { return at >= all_lo && at + n <= all_hi; }
};

// ---- tiles ----------------------------------------------------------------------------------

// A row of a head goes by pieces of 8 elements, 16 bytes.  Where its size is no multiple of 8 the last piece is the last 8 elements, which
// repeats some: products along a row need one side without them (Row), products across rows give them twice and one is stored.  Pieces behind the last one
// repeat the first.  So every load is 16 bytes of the row itself, wherever it starts; rows of fewer than 8 elements are taken one by one.
__device__ __forceinline__ uint32_t piece_at(uint32_t piece, uint32_t size) {
  return piece * 8u + 8u <= size ? piece * 8u : piece * 8u < size && size >= 8u ? size - 8u : 0u;
}
template <typename T>
__device__ __forceinline__ u32x4 load_piece(const T* row, uint32_t piece, uint32_t size) {
  Vec<T, 8> v;
  if (size >= 8u) load<false>(v, row + piece_at(piece, size));
  else load_end(v, row, size, 0.f);
  return u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
}
// How many elements at a piece's start are none of its own, and how many there are in front of its end (8, but for small sizes).
__device__ __forceinline__ void own_part(uint32_t piece, uint32_t size, uint32_t* begin, uint32_t* end) {
  const uint32_t left = piece * 8u < size ? size - piece * 8u : 0u;
  *begin = left >= 8u || size < 8u ? 0u : 8u - left, *end = size < 8u ? left : 8u;
}
template <typename T>
__device__ __forceinline__ const T* head_of(const Heads& x, uint32_t head) {
  return static_cast<const T*>(x.at) + (uint64_t)head * x.head;
}
template <typename T>
__device__ __forceinline__ const T* row_of(const T* head, const Heads& x, uint32_t row) {
  return head + (uint64_t)row * (uint32_t)x.row;
}

// kTile rows of D elements in LDS.  The 16-byte pieces of a row change places by the row's number: reads of one piece of 16 rows and
// transposing reads of four rows then meet every bank once.
constexpr int kTile = 64, kAhead = 4;  // kAhead: operands that are held, of which kAhead - 1 are on their way from LDS
template <int D>
__device__ __forceinline__ uint32_t turn(uint32_t row) {
  if constexpr (D == 64) return (row >> 1 & 1u) << 2 | (row >> 2 & 1u) << 1 | (row >> 3 & 1u);
  else return (row & 3u) << 2 | (row >> 2 & 3u);
}
// DIRECT: from memory to LDS without registers, where all rows start on 16 bytes; else through registers, at once, since those that hold a tile on its way are
// not to be had.  Rows behind the last one are the last one again: nobody sees them.
template <typename T, int D, int THREADS, bool DIRECT>
struct Stage {
  static constexpr int pieces = D / 8, loads = kTile * pieces / THREADS, step = THREADS / pieces;
  static_assert(step % 16 == 0, "rows that a thread loads turn their pieces alike");
  uint32_t at, row;     // DIRECT: this thread's first piece, in bytes behind the tile's first row, and from row to row
  const uint8_t* base;  // the next tile's first row, and how many are behind it
  uint32_t behind;
  // Tiles from row `first` on, one behind the other.
  __device__ __forceinline__ void set(const T* head, const Heads& x, uint32_t first, uint32_t rows, uint32_t size) {
    row = (uint32_t)x.row * 2u, base = reinterpret_cast<const uint8_t*>(row_of(head, x, first)), behind = rows - 1u - first;
    if constexpr (DIRECT) at = threadIdx.x / pieces * row + piece_at(threadIdx.x % pieces ^ turn<D>(threadIdx.x / pieces), size) * 2u;
  }
  __device__ __forceinline__ void fetch(uint8_t* tile, uint32_t size) {
    const uint32_t r = threadIdx.x / pieces;
    if constexpr (DIRECT) {
      uint8_t* to = tile + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024u;
      if (behind >= kTile - 1u) {
#pragma unroll
        for (uint32_t j = 0; j < loads; ++j) send_to_lds(base, at, j * step * row, to + j * THREADS * 16u);
      } else {
#pragma unroll
        for (uint32_t j = 0; j < loads; ++j) send_to_lds(base, at - r * row + min(r + j * step, behind) * row, 0, to + j * THREADS * 16u);
      }
    } else {
      u32x4 w[loads];
      const uint32_t piece = threadIdx.x % pieces;
#pragma unroll
      for (int j = 0; j < loads; ++j) w[j] = load_piece(reinterpret_cast<const T*>(base + (uint64_t)min(r + j * step, behind) * row), piece, size);
#pragma unroll
      for (int j = 0; j < loads; ++j) *reinterpret_cast<u32x4*>(tile + (r + j * step) * (D * 2) + (piece ^ turn<D>(r)) * 16u) = w[j];
    }
    base += (uint64_t)row * kTile, behind -= kTile;  // behind the last tile: of no concern
  }
};
// What this wavefront has fetched is in LDS, and everybody's is.
__device__ __forceinline__ void arrived() { wait_and_meet<0>(); }
// A lane's own row in registers, as an operand for all of k = 0 .. D - 1, zeros where there is no element.
template <typename T, int D>
struct Row {
  u32x4 w[D / 16];
  __device__ __forceinline__ void read(const T* row, uint32_t size) {
    const uint32_t half = (threadIdx.x & 63u) >> 5;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      const uint32_t piece = 2 * c + half;
      w[c] = load_piece(row, piece, size);
      if (size != D) {
        uint32_t begin, end;
        own_part(piece, size, &begin, &end);
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
          const uint32_t lo = 2 * e >= begin && 2 * e < end && piece * 8u < size ? 0xffffu : 0u, hi = 2 * e + 1 >= begin && 2 * e + 1 < end && piece * 8u < size ? 0xffff0000u : 0u;
          w[c][e] &= lo | hi;
        }
      }
    }
  }
  // Waits until it is there.  The compiler would wait where it is used first, in every round of a loop, and with it for the tiles that are on their way behind it
  // (16 heads of 8 192 rows of 128, both gradients 1 920 us for 1 780).
  __device__ __forceinline__ void wait() {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) asm volatile("" : "+v"(w[c]));
  }
};
template <int D>
struct Along {
  uint32_t at[D / 16];
  __device__ __forceinline__ void set() {
    const uint32_t lane = threadIdx.x & 63u, row = lane & 31u;
#pragma unroll
    for (uint32_t c = 0; c < D / 16; ++c) at[c] = row * (D * 2) + ((2u * c + (lane >> 5)) ^ turn<D>(row)) * 16u;
  }
  __device__ __forceinline__ u32x4 read(const uint8_t* tile, int sub, int c) const { return *reinterpret_cast<const u32x4*>(tile + sub * 32 * (D * 2) + at[c]); }
};
template <int D>
struct Across {
  uint32_t at[D / 32][2];
  __device__ __forceinline__ void set() {
    const uint32_t lane = threadIdx.x & 63u, i = lane & 15u, col = 16u * (lane >> 4 & 1u) + 4u * (i & 3u);
#pragma unroll
    for (uint32_t d = 0; d < D / 32; ++d)
#pragma unroll
      for (uint32_t e = 0; e < 2; ++e) {
        const uint32_t row = 8u * e + 4u * (lane >> 5) + i / 4u;
        at[d][e] = row * (D * 2) + ((d * 32u + col) / 8u ^ turn<D>(row)) * 16u + (i & 1u) * 8u;
      }
  }
  // Elements 32 d + l % 32 of the rows that a lane has of a score's column in elements 8 c .. 8 c + 7.
  __device__ __forceinline__ u32x4 read(const uint8_t* tile, int sub, int c, int d) const {
    const uint8_t* from = tile + (sub * 32 + c * 16) * (D * 2);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LMT_LDS s16x4*)(from + at[d][0]));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LMT_LDS s16x4*)(from + at[d][1]));
    const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
    return u32x4{a.x, a.y, b.x, b.y};
  }
};
// Column of scores as an operand.
template <typename T>
__device__ __forceinline__ u32x4 packed(const f32x16& x, int c) {
  return u32x4{pack2(T{}, x[8 * c], x[8 * c + 1]), pack2(T{}, x[8 * c + 2], x[8 * c + 3]), pack2(T{}, x[8 * c + 4], x[8 * c + 5]), pack2(T{}, x[8 * c + 6], x[8 * c + 7])};
}
template <typename T>
__device__ __forceinline__ void store_piece(T* row, uint32_t piece, const Vec<T, 8>& v, uint32_t size) {
  if (piece * 8u + 8u <= size) {
    store<false>(row + piece * 8u, v);
  } else if (piece * 8u < size) {
    uint32_t begin, end;
    own_part(piece, size, &begin, &end);
    T* to = row + piece_at(piece, size);
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e)
      if (e >= begin && e < end) store1(to + e, from_f32<T>(v.get(e)));
  }
}
// Sums whose column is the lane's row and whose rows are its elements, times `by`, to memory: the halves of a wavefront change places
// with what the other one has, so that each lane writes 8 neighbours.
template <typename T, int D>
__device__ __forceinline__ void store_row(T* row, const f32x16 (&x)[D / 32], float by, uint32_t size, bool here) {
  const uint32_t half = (threadIdx.x & 63u) >> 5;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pack2(T{}, x[d][8 * c + 2 * i] * by, x[d][8 * c + 2 * i + 1] * by);
      const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
      Vec<T, 8> v;
      v.w[0] = a[0], v.w[1] = b[0], v.w[2] = a[1], v.w[3] = b[1];
      if (here) store_piece(row, 4u * d + 2u * c + half, v, size);
    }
}
__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < kInf; }
template <int D>
__device__ __forceinline__ bool finite(const f32x16 (&x)[D / 32]) {
  float top = 0;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = __builtin_fmaf(x[d][i], 0.f, top);  // 0, or NaN
  return top == 0.f;
}

// ---- scores -----------------------------------------------------------------------------------

// Scores in units of log 2 from products.  PLAIN kernels: scale > 0 alone; others any scale, a cap and a slope.
// tanh(x) by its series up to 0.3, where its terms to x^9 leave 5e-8, else 1 - 2 / (e^2x + 1), which cancels near 0.  Scores
// are mostly far below their cap, so that a wavefront seldom needs the second form.
struct Score {
  float by, cap, to_cap, slope;  // by: scale * log2(e);  cap, slope: in units of log 2;  to_cap: scale / the cap
  __device__ __forceinline__ void set(const Attention& p, uint32_t head) {
    by = p.scale * kLog2e, cap = p.cap * kLog2e, to_cap = p.cap != 0.f ? p.scale / p.cap : 0.f;
    slope = p.slopes ? __uint_as_float(uniform(__float_as_uint(load1(p.slopes + head)))) * kLog2e : 0.f;  // here and now, as Row::wait
  }
  static __device__ __forceinline__ float series(float x) {
    const float y = x * x;
    float s = __builtin_fmaf(y, 0.021869488536f, -0.053968253968f);
    s = __builtin_fmaf(s, y, 0.133333333333f), s = __builtin_fmaf(s, y, -0.333333333333f);
    return __builtin_fmaf(s * y, x, x);
  }
  static __device__ __forceinline__ float tanh_of(float x) {
    const float e = exp2_of(__builtin_fabsf(x) * (2.f * kLog2e)), t = 1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f);
    return __builtin_fabsf(x) < 0.3f ? series(x) : __builtin_copysignf(t, x);
  }
  // N elements of a lane's column, from distance `apart` (the column's own row subtracted) on.  GRAD: d is multiplied by what the cap does to derivatives.
  template <int N, bool GRAD>
  __device__ __forceinline__ void of(f32x16 (&s)[N], float apart, f32x16 (&d)[N]) const {
    if (cap != 0.f) {
      float top = 0;
#pragma unroll
      for (int b = 0; b < N; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[b][e] *= to_cap, top = fmaxf(top, __builtin_fabsf(s[b][e]));
      if (any(!(top < 0.3f))) {
#pragma unroll
        for (int b = 0; b < N; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[b][e] = tanh_of(s[b][e]);
      } else {
#pragma unroll
        for (int b = 0; b < N; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[b][e] = series(s[b][e]);
      }
#pragma unroll
      for (int b = 0; b < N; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if constexpr (GRAD) d[b][e] *= __builtin_fmaf(-s[b][e], s[b][e], 1.f);
          s[b][e] *= cap;
        }
    } else {
#pragma unroll
      for (int b = 0; b < N; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[b][e] *= by;
    }
    if (slope != 0.f) {
#pragma unroll
      for (int b = 0; b < N; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[b][e] = __builtin_fmaf(-slope, __builtin_fabsf(apart + (float)(32 * b + 8 * (e / 4) + e % 4)), s[b][e]);
    }
  }
  // One score.
  __device__ __forceinline__ float of(float x, int apart, float* bend = nullptr) const {
    float y = x * by;
    if (bend) *bend = 1.f;
    if (cap != 0.f) {
      const float t = tanh_of(x * to_cap);
      y = cap * t;
      if (bend) *bend = __builtin_fmaf(-t, t, 1.f);
    }
    return slope != 0.f ? __builtin_fmaf(-slope, __builtin_fabsf((float)apart), y) : y;
  }
};

template <typename T>
__device__ __forceinline__ float dot(const T* x, const T* y, uint32_t size) {
  float s = 0;
  for (uint32_t d = 0; d < size; ++d) s = __builtin_fmaf(to_f32(load1(x + d)), to_f32(load1(y + d)), s);
  return s;
}

// fp16's range: weights are at most 2^kSlack, and 2^kShift times as large in fp16, so that the small ones lose fewer bits.
constexpr float kSlack = 8.f;
template <typename T>
constexpr float kShift = 0.f;
template <>
constexpr float kShift<_Float16> = 7.f;

// Which head and block of rows a workgroup has.  An XCD, which takes every eighth workgroup, has one head after the other, so that its L2 sees the
// same keys again and again.  CAUSAL, where blocks are from 1 to `tiles` long: the longest of all heads that an XCD has come first (kFirst or kLast says
// which end that is), since those that come last decide when it ends; heads that do not divide by XCDs go over all of them.
// 16 heads of 8 192 rows of 64: one head after the other 213 us, longest first 176.
enum Order { kAny, kFirst, kLast };
__device__ __forceinline__ void place(uint32_t tiles, uint32_t cuts, uint32_t lists, Order longest, uint32_t* tile, uint32_t* list) {
  constexpr uint32_t kXcds = 8;
  if (longest == kAny) {
    const uint32_t id = (uint32_t)neighbours(blockIdx.x, tiles * lists);
    *list = uniform(id / tiles), *tile = id - *list * tiles;
    return;
  }
  const uint32_t of_xcd = lists / kXcds;
  if (lists % kXcds == 0) {
    const uint32_t in_xcd = blockIdx.x / kXcds;
    *tile = uniform(in_xcd / of_xcd), *list = blockIdx.x % kXcds * of_xcd + in_xcd - *tile * of_xcd;
  } else {
    *tile = uniform(blockIdx.x / lists), *list = blockIdx.x - *tile * lists;
  }
  if (longest == kLast && *tile >= cuts) *tile = tiles - 1u - (*tile - cuts);
}

// Scores that the column's row does not see, its first element `from` places into what it sees: none.  Their weights are 0, and so are
// weights times what is finite; what is not shows in the sums.
__device__ __forceinline__ void hide(f32x16& s, uint32_t from, uint32_t n) {
#pragma unroll
  for (int e = 0; e < 16; ++e) s[e] = from + (uint32_t)(8 * (e / 4) + e % 4) < n ? s[e] : -kInf;
}
__device__ __forceinline__ float largest(const f32x16 (&s)[2]) {
  float top[2] = {s[0][0], s[1][0]};
#pragma unroll
  for (int e = 1; e < 16; ++e) top[0] = fmaxf(top[0], s[0][e]), top[1] = fmaxf(top[1], s[1][e]);
  return fmaxf(top[0], top[1]);
}

// ---- forward ------------------------------------------------------------------------------------

// One row, a wavefront: only of what the row sees, so that infinities and NaN elsewhere stay there.  Slow: with loads of 2 bytes a lane, rows of a wavefront one after the
// other, and every row that rightly sees an infinity or a NaN comes here too.  One NaN that 8 192 rows of 16 heads see: of 64, all see all, 211 ms instead of 0.38, the gradients 349 (grad_q_row,
// grad_kv_row) instead of 1.2; of 128, causal, 204 and 444.  From there on it grows with the square of a sequence, below with its length (73 and 108 ms at 4 096 rows, 15 and 24 at 1 024).
template <typename T>
__device__ __forceinline__ void attend_row(const Attention& p, uint32_t head, uint32_t kv, uint32_t i, int lo, int hi) {
  const uint32_t lane = threadIdx.x & 63u;
  const T *k = head_of<T>(p.k, kv), *v = head_of<T>(p.v, kv), *q = row_of(head_of<T>(p.q, head), p.q, i);
  Score score;
  score.set(p, head);
  float m = -kInf, l = 0, o[2] = {};
  for (int j0 = lo; j0 < hi; j0 += 64) {
    const int j = j0 + (int)lane;
    float s = -kInf;
    if (j < hi) s = score.of(dot(q, row_of(k, p.k, (uint32_t)j), p.size), abs((int)i - j));
    const float top = fmaxf(m, wave_max(s)), base = top == -kInf ? 0.f : top;
    const float w = j < hi ? exp2_of(s - base) : 0.f, by = m == -kInf ? 0.f : exp2_of(m - base);
    m = top, l = __builtin_fmaf(l, by, wave_sum(w)), o[0] *= by, o[1] *= by;
    for (int n = 0; n < min(64, hi - j0); ++n) {
      const float x = __shfl(w, n);
      const T* row = row_of(v, p.v, (uint32_t)(j0 + n));
#pragma unroll
      for (uint32_t e = 0; e < 2; ++e)
        if (lane + 64u * e < p.size) o[e] = __builtin_fmaf(x, to_f32(load1(row + lane + 64u * e)), o[e]);
    }
  }
  T* out = const_cast<T*>(row_of(head_of<T>(p.out, head), p.out, i));
#pragma unroll
  for (uint32_t e = 0; e < 2; ++e)
    if (lane + 64u * e < p.size) store1(out + lane + 64u * e, from_f32<T>(l == 0.f ? 0.f : o[e] / l));
  if (p.lse && lane == 0) store1(p.lse + (uint64_t)head * p.rows + i, l == 0.f ? -kInf : (m + __builtin_amdgcn_logf(l)) * kLn2);
}

// The scores of the next tile are made while those of this one go through exp2: matrix instructions and the others take turns in the
// instruction stream, as one wavefront's do not overlap unless they are side by side in it.  Operands are asked for kAhead - 1 instructions early.
// A tile of 32 x 64 is 16 matrix instructions of 32 cycles with heads of 64 (32 with 128) and about 200 others, an exponential counting double, so that heads of 64 are
// bound by vector issue (78 % of the busy cycles; matrix cores 45 %) and heads of 128 by the two together (53 and 56 %).  LDS has no bank conflicts.  bf16, 16 heads
// of 8 192 rows: 64, causal 176 us, 0.78 PFLOP/s; 128 512 us, 1.07, causal 282, 0.97, with a cap 368 (its tanh is as many instructions again).  16 sequences of 512, heads of 64: 34 us.
// One workgroup's 64 keys take 0.93 us (64) or 1.18 (128), which is what few rows wait for.  Three workgroups a compute unit with heads of 64: 118 us where two take 146
// (128 sequences of up to 512, 16 heads).  Two tiles to a round instead of one: 1.18 -> 1.07 us, but registers spill and 16 of 512 take 39 us for 34.
template <typename T, int D, bool PLAIN, bool DIRECT>
__global__ __launch_bounds__(kThreads, D == 64 && DIRECT ? 3 : 2) void k_attend(const Attention p, uint32_t tiles) {
  __shared__ __align__(16) uint8_t keys[2][kTile * D * 2], values[2][kTile * D * 2];
  __shared__ Seen seen;
  uint32_t tile, head;
  place(tiles, p.cuts, p.heads, p.causal ? kLast : kAny, &tile, &head);
  Block block;
  block.set(p, tile);
  const uint32_t kv = uniform(head / p.group), wave = threadIdx.x >> 6, lane = threadIdx.x & 63u, row = wave * 32u + (lane & 31u), i = (uint32_t)block.first + row;
  const T *k = head_of<T>(p.k, kv), *v = head_of<T>(p.v, kv);
  check_sequences(p);
  Row<T, D> q;
  q.read(row_of(head_of<T>(p.q, head), p.q, min(i, p.rows - 1u)), p.size);
  find_seen<false>(p, block, seen);
  Span span;
  span.read(seen, row);
  const int first = __builtin_amdgcn_readfirstlane(seen.first), last = __builtin_amdgcn_readfirstlane(seen.last);
  Score score;
  score.set(p, head);
  Along<D> along;
  Across<D> across;
  along.set(), across.set();
  float m = -kInf, top = -kInf, sum[4] = {};
  f32x16 o[D / 32] = {}, s[2];
  Stage<T, D, kThreads, DIRECT> next_k, next_v;
  // The scores of tile `at`, in buffer `now`, become weights, and those of the tile behind it are made.
  const auto pass = [&](int at, uint32_t now) {
    const bool more = at + kTile < last, more_keys = at + 2 * kTile < last;
    if (more_keys) next_k.fetch(keys[now], p.size);
    if (more) next_v.fetch(values[now ^ 1u], p.size);
    if (span.touches(at, kTile)) {
      const int j0 = at + 4 * (int)(lane >> 5);
      const bool inside = span.inside(at, kTile);
      if constexpr (!PLAIN) score.of<2, false>(s, (float)(j0 - (int)i), s);
      if (!inside) {
        const uint32_t from = (uint32_t)(j0 - span.lo), n = (uint32_t)(span.hi - span.lo);
        hide(s[0], from, n), hide(s[1], from + 32u, n);
      }
      if (!PLAIN || !inside) top = largest(s);
      float most = halves_max(top);
      if constexpr (PLAIN) most *= score.by;
      if (any(most > m + kSlack)) {
        const float up = fmaxf(m, most), by = m == -kInf ? 0.f : exp2_of(m - up);
        m = up;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] *= by;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] *= by;
      }
      const float base = (m == -kInf ? 0.f : m) - kShift<T>;
      u32x4 w[2][2], ahead[kAhead];
      constexpr int kSteps = 2 * (D / 16), kEach = 32 / kSteps;  // instructions of either kind; elements between two
      // operand t: of the next scores, then of this tile's values
      const auto operand = [&](int t) {
        if (t < kSteps) return along.read(keys[now ^ 1u], t % 2, t / 2);  // behind the last tile: of no concern
        const int u = t - kSteps, of = u / (D / 32);
        return across.read(values[now], of / 2, of % 2, u % (D / 32));
      };
      f32x16 next[2] = {};
      float tops[2];
#pragma unroll
      for (int t = 0; t < kAhead - 1; ++t) ahead[t] = operand(t);
      each<2 * kSteps>([&](auto number) {
        constexpr int t = decltype(number)::value;
        if (t + kAhead - 1 < 2 * kSteps) ahead[(t + kAhead - 1) % kAhead] = operand(t + kAhead - 1);
        if constexpr (t < kSteps) {
          next[t % 2] = mma(T{}, ahead[t % kAhead], q.w[t / 2], next[t % 2]);
#pragma unroll
          for (int e = t * kEach; e < (t + 1) * kEach; ++e) {
            const float x = exp2_of(PLAIN ? __builtin_fmaf(s[e / 16][e % 16], score.by, -base) : s[e / 16][e % 16] - base);
            s[e / 16][e % 16] = x, sum[e % 4] += x;
          }
          if constexpr ((t + 1) * kEach % 8 == 0) w[((t + 1) * kEach - 8) / 16][((t + 1) * kEach - 8) / 8 % 2] = packed<T>(s[((t + 1) * kEach - 8) / 16], ((t + 1) * kEach - 8) / 8 % 2);
        } else {
          constexpr int u = t - kSteps, of = u / (D / 32), d = u % (D / 32);
          o[d] = mma(T{}, ahead[t % kAhead], w[of / 2][of % 2], o[d]);
          if constexpr (u >= kSteps / 2) {  // the next scores, which are there by now, move, and the largest is found
            constexpr int b = (u - kSteps / 2) * 64 / kSteps / 16, n = 64 / kSteps, e0 = (u - kSteps / 2) * n % 16;
#pragma unroll
            for (int e = e0; e < e0 + n; ++e) {
              float x = next[b][e];
              asm volatile("" : "+v"(x));  // here, and not behind the last product
              s[b][e] = x, tops[b] = e == 0 ? x : fmaxf(tops[b], x);
            }
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (PLAIN) top = fmaxf(tops[0], tops[1]);
    } else if (more && span.touches(at + kTile, kTile)) {
      s[0] = s[1] = f32x16{};
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int b = 0; b < 2; ++b) s[b] = mma(T{}, along.read(keys[now ^ 1u], b, c), q.w[c], s[b]);
      if constexpr (PLAIN) top = largest(s);
    }
    arrived();
  };
  if (first < last) {
    next_k.set(k, p.k, (uint32_t)first, p.rows, p.size), next_v.set(v, p.v, (uint32_t)first, p.rows, p.size);
    next_k.fetch(keys[0], p.size), next_v.fetch(values[0], p.size);
    arrived();
    const bool more = first + kTile < last;
    if (more) next_k.fetch(keys[1], p.size);
    s[0] = s[1] = f32x16{};
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
      for (int b = 0; b < 2; ++b) s[b] = mma(T{}, along.read(keys[0], b, c), q.w[c], s[b]);
    if constexpr (PLAIN) top = largest(s);
    arrived();
    uint32_t now = 0;
    for (int at = first; at < last; at += kTile, now ^= 1u) pass(at, now);
  }
  float l = (sum[0] + sum[1]) + (sum[2] + sum[3]);
  l = halves_sum(l);
  const bool some = span.some();
  const bool again = some && !(finite<D>(o) && finite(l));
  const uint64_t rows_again = __builtin_amdgcn_ballot_w64(again);
  const uint32_t redo = (uint32_t)rows_again | (uint32_t)(rows_again >> 32);
  const bool mine = span.mine() && !(redo >> (lane & 31u) & 1u);
  if (!some || l == 0.f) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = f32x16{};
    l = 0.f;
  }
  store_row<T, D>(const_cast<T*>(row_of(head_of<T>(p.out, head), p.out, min(i, p.rows - 1u))), o, l == 0.f ? 0.f : 1.f / l, p.size, mine);
  if (p.lse && mine && lane < 32u) store1(p.lse + (uint64_t)head * p.rows + i, l == 0.f ? -kInf : (m - kShift<T> + __builtin_amdgcn_logf(l)) * kLn2);
  for (uint32_t left = redo; left; left &= left - 1u) {
    const uint32_t r = wave * 32u + (uint32_t)__builtin_ctz(left);
    attend_row<T>(p, head, kv, (uint32_t)block.first + r, seen.lo[r], seen.hi[r]);
  }
}

// ---- gradient -------------------------------------------------------------------------------------

// What d are multiplied by before they are rounded to fp16: a power of two of the lane's own row (of q, or of k), that brings the largest so far to
// between 2^13 and 2^14 when it has left fp16's range, so that others are exact to 2^-38 of it; the row's sums, which are the lane's too, follow.  Rows of
// the same wavefront that have come beyond 2^14 go with it, which halves how often that happens (9 of 256 half tiles instead of 21 for normal numbers).  One power for all rows of a
// wavefront would cost less (16 heads of 8 192 rows of 128 in fp16: 2 072 us for 2 098), but take bits, or everything, from rows beside one with much larger d, in another sequence or in none.  Lanes
// whose row sees nothing have no scale: in tiles that are inside of all others' intervals their d are not hidden, and grow with whatever the rows hold.  What is
// not finite has none either: its sums are not, and are computed once more.  bf16 has fp32's range.
constexpr float kHalfMost = 65504.f;
template <typename T>
struct Range {
  float by = 1.f;
  __device__ __forceinline__ void begin() {
    if constexpr (sizeof(T) == 2 && kShift<T> != 0.f) by = 0x1p60f;
  }
  // Where x, times by, are too large: then `by` is smaller, x and the sums have followed.
  template <int N, int M>
  __device__ __forceinline__ void fit(f32x16 (&x)[N], f32x16 (&sums)[M], bool some) {
    if constexpr (kShift<T> != 0.f) {
      float top = 0;
#pragma unroll
      for (int b = 0; b < N; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, __builtin_fabsf(x[b][e]));
      if (any(some && top > kHalfMost)) {
        top = halves_max(top);
        const float down = some && top >= 0x1p14f && top < kInf ? __uint_as_float((127u + 13u + 127u - (__float_as_uint(top) >> 23)) << 23) : 1.f;
        by *= down;
#pragma unroll
        for (int b = 0; b < N; ++b) x[b] *= down;
#pragma unroll
        for (int b = 0; b < M; ++b) sums[b] *= down;
      }
    }
  }
};

// Row i's gradient of q, a wavefront.
template <typename T>
__device__ __forceinline__ void grad_q_row(const Attention& p, uint32_t head, uint32_t kv, uint32_t i, int lo, int hi, float lse, float delta) {
  const uint32_t lane = threadIdx.x & 63u;
  const T *k = head_of<T>(p.k, kv), *v = head_of<T>(p.v, kv), *q = row_of(head_of<T>(p.q, head), p.q, i), *go = row_of(head_of<T>(p.grad_out, head), p.grad_out, i);
  Score score;
  score.set(p, head);
  float sum[2] = {};
  for (int j0 = lo; j0 < hi; j0 += 64) {
    const int j = j0 + (int)lane;
    float d = 0;
    if (j < hi) {
      float bend;
      const float s = score.of(dot(q, row_of(k, p.k, (uint32_t)j), p.size), abs((int)i - j), &bend);
      d = exp2_of(s - lse) * (dot(go, row_of(v, p.v, (uint32_t)j), p.size) - delta) * bend;
    }
    for (int n = 0; n < min(64, hi - j0); ++n) {
      const float x = __shfl(d, n);
      const T* row = row_of(k, p.k, (uint32_t)(j0 + n));
#pragma unroll
      for (uint32_t e = 0; e < 2; ++e)
        if (lane + 64u * e < p.size) sum[e] = __builtin_fmaf(x, to_f32(load1(row + lane + 64u * e)), sum[e]);
    }
  }
  T* to = const_cast<T*>(row_of(head_of<T>(p.grad_q, head), p.grad_q, i));
#pragma unroll
  for (uint32_t e = 0; e < 2; ++e)
    if (lane + 64u * e < p.size) store1(to + lane + 64u * e, from_f32<T>(sum[e] * p.scale));
}

// lse in units of log 2, as what is subtracted from scores: a row without weights has none.
__device__ __forceinline__ float subtracted(float lse) { return lse == -kInf ? kInf : lse * kLog2e; }

// Gradient of q and, for the next kernel, delta = grad_out . out of every row: as the forward pass, scores and products with v from a tile of each, d into the
// sums with k across.  One half tile's exponentials stand beside the other one's products.  Three products here and four in the next kernel instead of five in
// one: sums of both kinds do not fit a wavefront's registers, and one kernel would have to add one of them to memory from many workgroups, in no order.  16 heads of 8 192 rows
// of 128, causal: 386 us, matrix cores busy 67 % of the time; 128 sequences of up to 512, 16 heads of 64: 155.  (The general form of heads of 128 keeps 20 bytes in
// scratch, 28 to 32 where rows cannot go straight to LDS: with an operand less ahead it does not, and takes 297 us for 281.  All other forms keep nothing there, but for
// k_attend_grad_kv's general one of heads of 64 in bf16: 48 bytes, 24 where rows cannot go straight.)
template <typename T, int D, bool PLAIN, bool DIRECT>
__global__ __launch_bounds__(kThreads, 2) void k_attend_grad_q(const Attention p, uint32_t tiles) {
  __shared__ __align__(16) uint8_t keys[2][kTile * D * 2], values[2][kTile * D * 2];
  __shared__ Seen seen;
  uint32_t tile, head;
  place(tiles, 0u, p.heads, p.causal ? kLast : kAny, &tile, &head);
  const Block block{(int)(tile * kRows), -1};
  const uint32_t kv = uniform(head / p.group), wave = threadIdx.x >> 6, lane = threadIdx.x & 63u, row = wave * 32u + (lane & 31u), i = (uint32_t)block.first + row, held = min(i, p.rows - 1u);
  const T *k = head_of<T>(p.k, kv), *v = head_of<T>(p.v, kv);
  check_sequences(p);
  Row<T, D> q, go;
  q.read(row_of(head_of<T>(p.q, head), p.q, held), p.size), go.read(row_of(head_of<T>(p.grad_out, head), p.grad_out, held), p.size);
  float delta = 0;
  {
    Row<T, D> out;
    out.read(row_of(head_of<T>(p.out, head), p.out, held), p.size);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      const Vec<T, 8> a = __builtin_bit_cast(Vec<T, 8>, out.w[c]), b = __builtin_bit_cast(Vec<T, 8>, go.w[c]);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = __builtin_fmaf(a.get(e), b.get(e), delta);
    }
    delta = halves_sum(delta);
  }
  const float lse = subtracted(load1(p.lse + (uint64_t)head * p.rows + held));
  find_seen<false>(p, block, seen);
  q.wait(), go.wait();
  Span span;
  span.read(seen, row);
  const bool some = span.some();
  if (span.mine() && lane < 32u) store1(p.delta + (uint64_t)head * p.rows + i, delta);
  const int first = __builtin_amdgcn_readfirstlane(seen.first), last = __builtin_amdgcn_readfirstlane(seen.last);
  Score score;
  score.set(p, head);
  Along<D> along;
  Across<D> across;
  along.set(), across.set();
  Range<T> range;
  range.begin();
  f32x16 sum[D / 32] = {};
  Stage<T, D, kThreads, DIRECT> next_k, next_v;
  if (first < last) {
    next_k.set(k, p.k, (uint32_t)first, p.rows, p.size), next_v.set(v, p.v, (uint32_t)first, p.rows, p.size);
    next_k.fetch(keys[0], p.size), next_v.fetch(values[0], p.size);
  }
  arrived();
  uint32_t now = 0;
  for (int at = first; at < last; at += kTile, now ^= 1u) {
    const bool more = at + kTile < last;
    if (more) next_k.fetch(keys[now ^ 1u], p.size), next_v.fetch(values[now ^ 1u], p.size);
    if (span.touches(at, kTile)) {
      {
        constexpr int kHalf = D / 16, kSteps = 6 * kHalf, kAhead = 3;  // of k; of matrix instructions: scores and products with v of either half, then sums of either
        f32x16 s[2][1] = {}, dp[2][1] = {};
        u32x4 w[2][2], ahead[kAhead];
        const auto operand = [&](int t) {
          if (t < 4 * kHalf) return along.read(t % 2 ? values[now] : keys[now], t / (2 * kHalf), t / 2 % kHalf);
          const int u = t - 4 * kHalf, b = u / kHalf, of = u % kHalf;
          return across.read(keys[now], b, of / (D / 32), of % (D / 32));
        };
        const uint32_t from = (uint32_t)(at + 4 * (int)(lane >> 5) - span.lo), n = (uint32_t)(span.hi - span.lo);
        const bool inside = span.inside(at, kTile);
        const auto element = [&](int b, int e) {
          const float x = exp2_of(PLAIN ? __builtin_fmaf(s[b][0][e], score.by, -lse) : s[b][0][e] - lse);
          s[b][0][e] = (PLAIN ? __builtin_fmaf(dp[b][0][e], range.by, -delta * range.by) : dp[b][0][e]) * x;
        };
        const auto general = [&](auto half_of) {  // what is not PLAIN's, for a whole half
          constexpr int b = decltype(half_of)::value;
#pragma unroll
          for (int e = 0; e < 16; ++e) dp[b][0][e] = __builtin_fmaf(dp[b][0][e], range.by, -delta * range.by);
          score.of<1, true>(s[b], (float)(at + 32 * b + 4 * (int)(lane >> 5) - (int)i), dp[b]);
        };
#pragma unroll
        for (int t = 0; t < kAhead - 1; ++t) ahead[t] = operand(t);
        each<kSteps>([&](auto number) {
          constexpr int t = decltype(number)::value;
          if (t + kAhead - 1 < kSteps) ahead[(t + kAhead - 1) % kAhead] = operand(t + kAhead - 1);
          if constexpr (t < 4 * kHalf) {
            constexpr int b = t / (2 * kHalf), c = t / 2 % kHalf;
            if (t % 2) dp[b][0] = mma(T{}, ahead[t % kAhead], go.w[c], dp[b][0]);
            else s[b][0] = mma(T{}, ahead[t % kAhead], q.w[c], s[b][0]);
          } else {
            constexpr int u = t - 4 * kHalf, b = u / kHalf, of = u % kHalf, d = of % (D / 32);
            sum[d] = mma(T{}, ahead[t % kAhead], w[b][of / (D / 32)], sum[d]);
          }
          // the first half's elements beside the second half's scores, the second half's beside the first one's sums
          if constexpr (!PLAIN) {
            if constexpr (t == 2 * kHalf || t == 4 * kHalf) general(std::integral_constant<int, t / (2 * kHalf) - 1>{});
          }
          if constexpr (t == 2 * kHalf || t == 4 * kHalf) {
            if (!inside) hide(s[t / (2 * kHalf) - 1][0], from + (t == 4 * kHalf ? 32u : 0u), n);
          }
          if constexpr (t >= 2 * kHalf && t < 5 * kHalf) {
            constexpr int b = t >= 4 * kHalf, n_steps = b ? kHalf : 2 * kHalf, step = b ? t - 4 * kHalf : t - 2 * kHalf;
#pragma unroll
            for (int e = step * 16 / n_steps; e < (step + 1) * 16 / n_steps; ++e) element(b, e);
            if constexpr (step + 1 == n_steps) {
              range.fit(s[b], sum, some);
              w[b][0] = packed<T>(s[b][0], 0), w[b][1] = packed<T>(s[b][0], 1);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        });
      }
    }
    arrived();
  }
  const uint64_t rows_again = __builtin_amdgcn_ballot_w64(some && !finite<D>(sum));
  const uint32_t redo = (uint32_t)rows_again | (uint32_t)(rows_again >> 32);
  if (!some) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) sum[d] = f32x16{};
  }
  store_row<T, D>(const_cast<T*>(row_of(head_of<T>(p.grad_q, head), p.grad_q, held)), sum, p.scale / range.by, p.size, span.mine() && !(redo >> (lane & 31u) & 1u));
  for (uint32_t left = redo; left; left &= left - 1u) {
    const int b = __builtin_ctz(left);
    const uint32_t r = wave * 32u + (uint32_t)b;
    grad_q_row<T>(p, head, kv, (uint32_t)block.first + r, seen.lo[r], seen.hi[r], __shfl(lse, b), __shfl(delta, b));
  }
}

// Where the gradients of a key go: the tensors, or a part's sums.
template <typename T, int D>
__device__ __forceinline__ void store_key(const Attention& p, const Heads& to, float* part, uint32_t kv, uint32_t j, const f32x16 (&x)[D / 32], float by, bool here) {
  if (p.parts == 1u) {
    store_row<T, D>(const_cast<T*>(row_of(head_of<T>(to, kv), to, min(j, p.rows - 1u))), x, by, p.size, here);
    return;
  }
  if (!here) return;
  float* row = part + ((uint64_t)kv * p.rows + j) * D + 4u * ((threadIdx.x & 63u) >> 5);
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(LMT_GLOBAL f32x4*)(row + 32 * d + 8 * g) = f32x4{x[d][4 * g] * by, x[d][4 * g + 1] * by, x[d][4 * g + 2] * by, x[d][4 * g + 3] * by};
}

// Key j's gradients from query heads [h0, h1), a wavefront.
template <typename T, int D>
__device__ __forceinline__ void grad_kv_row(const Attention& p, uint32_t kv, uint32_t h0, uint32_t h1, uint32_t j, int lo, int hi, float* part_k, float* part_v) {
  const uint32_t lane = threadIdx.x & 63u;
  const T *k = row_of(head_of<T>(p.k, kv), p.k, j), *v = row_of(head_of<T>(p.v, kv), p.v, j);
  float dk[2] = {}, dv[2] = {};
  for (uint32_t head = h0; head < h1; ++head) {
    const T *q = head_of<T>(p.q, head), *go = head_of<T>(p.grad_out, head);
    Score score;
    score.set(p, head);
    for (int i0 = lo; i0 < hi; i0 += 64) {
      const int i = i0 + (int)lane;
      float w = 0, d = 0;
      if (i < hi) {
        float bend;
        const uint64_t at = (uint64_t)head * p.rows + (uint32_t)i;
        w = exp2_of(score.of(dot(row_of(q, p.q, (uint32_t)i), k, p.size), abs(i - (int)j), &bend) - subtracted(load1(p.lse + at)));
        d = w * (dot(row_of(go, p.grad_out, (uint32_t)i), v, p.size) - load1(p.delta + at)) * bend;
      }
      for (int n = 0; n < min(64, hi - i0); ++n) {
        const float x = __shfl(d, n), y = __shfl(w, n);
        const T *a = row_of(q, p.q, (uint32_t)(i0 + n)), *b = row_of(go, p.grad_out, (uint32_t)(i0 + n));
#pragma unroll
        for (uint32_t e = 0; e < 2; ++e)
          if (lane + 64u * e < p.size) {
            dk[e] = __builtin_fmaf(x, to_f32(load1(a + lane + 64u * e)), dk[e]);
            dv[e] = __builtin_fmaf(y, to_f32(load1(b + lane + 64u * e)), dv[e]);
          }
      }
    }
  }
#pragma unroll
  for (uint32_t e = 0; e < 2; ++e) {
    const uint32_t c = lane + 64u * e;
    if (c >= p.size) continue;
    if (p.parts == 1u) {
      store1(const_cast<T*>(row_of(head_of<T>(p.grad_k, kv), p.grad_k, j)) + c, from_f32<T>(dk[e] * p.scale));
      store1(const_cast<T*>(row_of(head_of<T>(p.grad_v, kv), p.grad_v, j)) + c, from_f32<T>(dv[e]));
    } else {
      const uint32_t in = c / 8u * 8u + 8u <= p.size || p.size < 8u ? c : c + 8u - p.size % 8u;  // the last piece ends with the row
      store1(part_k + ((uint64_t)kv * p.rows + j) * D + in, dk[e] * p.scale);
      store1(part_v + ((uint64_t)kv * p.rows + j) * D + in, dv[e]);
    }
  }
}

// Gradients of k and v: a lane has a key, the rows that see it come by in tiles, for one query head after the other.  Scores as Q K^T, so that
// what a lane has of them is an operand of dO^T P and Q^T d.  With heads of 128 the sums and the key's rows take more than half the registers: one wavefront a SIMD, and
// what its instructions wait for each other is not filled by another's: 16 heads of 8 192 rows of 128, causal 600 us, matrix cores busy 45 % of the time, vector issue 35 %, 31 % waiting
// (operands 5 or 7 instructions early instead of 3: no difference).  Heads of 64, two wavefronts: 128 sequences of up to 512, 16 heads 204 us.
template <typename T, int D, bool PLAIN, bool DIRECT>
__global__ __launch_bounds__(kThreads, D == 64 ? 2 : 1) void k_attend_grad_kv(const Attention p, uint32_t tiles) {
  __shared__ __align__(16) uint8_t queries[2][kTile * D * 2], grads[2][kTile * D * 2];
  __shared__ __align__(16) float lse[2][kTile], delta[2][kTile];
  __shared__ Seen seen;
  uint32_t tile, list;
  place(tiles, 0u, p.kv_heads * p.parts, p.causal ? kFirst : kAny, &tile, &list);
  const Block block{(int)(tile * kRows), -1};
  const uint32_t kv = uniform(list / p.parts), part = list - kv * p.parts, h0 = kv * p.group + uniform(part * p.group / p.parts), h1 = kv * p.group + uniform((part + 1u) * p.group / p.parts);
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u, row = wave * 32u + (lane & 31u), j = (uint32_t)block.first + row, held = min(j, p.rows - 1u);
  Row<T, D> k, v;
  k.read(row_of(head_of<T>(p.k, kv), p.k, held), p.size), v.read(row_of(head_of<T>(p.v, kv), p.v, held), p.size);
  find_seen<true>(p, block, seen);
  k.wait(), v.wait();
  Span span;
  span.read(seen, row);
  const bool some = span.some();
  const int first = __builtin_amdgcn_readfirstlane(seen.first), last = __builtin_amdgcn_readfirstlane(seen.last);
  Along<D> along;
  Across<D> across;
  along.set(), across.set();
  Range<T> range;
  range.begin();
  f32x16 dk[D / 32] = {}, dv[D / 32] = {};
  Stage<T, D, kThreads, DIRECT> next_q, next_go;
  float next_lse = 0, next_delta = 0;
  const auto fetch = [&](uint32_t head, int at, uint32_t to) {
    if (at == first) next_q.set(head_of<T>(p.q, head), p.q, (uint32_t)first, p.rows, p.size), next_go.set(head_of<T>(p.grad_out, head), p.grad_out, (uint32_t)first, p.rows, p.size);
    next_q.fetch(queries[to], p.size), next_go.fetch(grads[to], p.size);
    if (threadIdx.x < kTile) {
      const uint64_t from = (uint64_t)head * p.rows + min((uint32_t)at + threadIdx.x, p.rows - 1u);
      next_lse = load1(p.lse + from), next_delta = load1(p.delta + from);
    }
  };
  const auto put = [&](uint32_t to) {
    if (threadIdx.x < kTile) lse[to][threadIdx.x] = subtracted(next_lse), delta[to][threadIdx.x] = next_delta;
  };
  if (first < last) fetch(h0, first, 0), put(0);
  arrived();
  uint32_t now = 0;
  for (uint32_t head = h0; first < last && head < h1; ++head) {
    Score score;
    score.set(p, head);
    for (int at = first; at < last; at += kTile, now ^= 1u) {
      const bool wrap = at + kTile >= last, more = !wrap || head + 1u < h1;
      if (more) fetch(wrap ? head + 1u : head, wrap ? first : at + kTile, now ^ 1u);
      if (span.touches(at, kTile)) {
        {
          constexpr int kHalf = D / 16, kSteps = 8 * kHalf, kAhead = D == 128 ? 4 : PLAIN ? 3 : 2;
          f32x16 s[2][1] = {}, d[2][1] = {};
          u32x4 w[2][2], x[2][2], ahead[kAhead];
          constexpr int kRowsAhead = D == 64 ? 1 : 2;  // registers are short
          f32x4 less[kRowsAhead], dots[kRowsAhead];    // of four rows, and of the next four
          const int half = 4 * (int)(lane >> 5);
          const auto rows = [&](int b, int g) {
            less[g % kRowsAhead] = *reinterpret_cast<const f32x4*>(&lse[now][32 * b + 8 * g + half]), dots[g % kRowsAhead] = *reinterpret_cast<const f32x4*>(&delta[now][32 * b + 8 * g + half]);
          };
          const auto operand = [&](int t) {
            if (t < 4 * kHalf) return along.read(t % 2 ? grads[now] : queries[now], t / (2 * kHalf), t / 2 % kHalf);
            const int u = t - 4 * kHalf, b = u / (2 * kHalf), of = u / 2 % kHalf;
            return across.read(u % 2 ? queries[now] : grads[now], b, of / (D / 32), of % (D / 32));
          };
          const uint32_t from = (uint32_t)(at + half - span.lo), n = (uint32_t)(span.hi - span.lo);
          const bool inside = span.inside(at, kTile);
          const auto element = [&](int b, int e) {
            const int g = e / 4;
            float p_ = exp2_of(PLAIN ? __builtin_fmaf(s[b][0][e], score.by, -less[g % kRowsAhead][e % 4]) : s[b][0][e] - less[g % kRowsAhead][e % 4]);
            const float d_ = (PLAIN ? __builtin_fmaf(d[b][0][e], range.by, -dots[g % kRowsAhead][e % 4] * range.by) : d[b][0][e]) * p_;
            if constexpr (kShift<T> != 0.f) p_ *= 0x1p14f;  // weights are at most 1
            s[b][0][e] = p_, d[b][0][e] = d_;
          };
          const auto general = [&](auto half_of) {  // what is not PLAIN's, for a whole half
            constexpr int b = decltype(half_of)::value;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const f32x4 x = *reinterpret_cast<const f32x4*>(&delta[now][32 * b + 8 * g + half]);
#pragma unroll
              for (int r = 0; r < 4; ++r) d[b][0][4 * g + r] = __builtin_fmaf(d[b][0][4 * g + r], range.by, -x[r] * range.by);
            }
            score.of<1, true>(s[b], (float)(at + 32 * b + half - (int)j), d[b]);
          };
#pragma unroll
          for (int t = 0; t < kAhead - 1; ++t) ahead[t] = operand(t);
          each<kSteps>([&](auto number) {
            constexpr int t = decltype(number)::value;
            if (t + kAhead - 1 < kSteps) ahead[(t + kAhead - 1) % kAhead] = operand(t + kAhead - 1);
            if constexpr (t < 4 * kHalf) {
              constexpr int b = t / (2 * kHalf), c = t / 2 % kHalf;
              if (t % 2) d[b][0] = mma(T{}, ahead[t % kAhead], v.w[c], d[b][0]);
              else s[b][0] = mma(T{}, ahead[t % kAhead], k.w[c], s[b][0]);
            } else {
              constexpr int u = t - 4 * kHalf, b = u / (2 * kHalf), of = u / 2 % kHalf, e = of % (D / 32);
              if (u % 2) dk[e] = mma(T{}, ahead[t % kAhead], x[b][of / (D / 32)], dk[e]);
              else dv[e] = mma(T{}, ahead[t % kAhead], w[b][of / (D / 32)], dv[e]);
            }
            if constexpr (!PLAIN) {
              if constexpr (t == 2 * kHalf || t == 4 * kHalf) general(std::integral_constant<int, t / (2 * kHalf) - 1>{});
            }
            if constexpr (t == 2 * kHalf || t == 4 * kHalf) {
              if (!inside) hide(s[t / (2 * kHalf) - 1][0], from + (t == 4 * kHalf ? 32u : 0u), n);
            }
            if constexpr (t == 2 * kHalf - 1 && kRowsAhead == 2) rows(0, 0);
            if constexpr (t >= 2 * kHalf && t < 6 * kHalf) {
              constexpr int b = t >= 4 * kHalf, step = t - (b ? 4 : 2) * kHalf;
#pragma unroll
              for (int e = step * 8 / kHalf; e < (step + 1) * 8 / kHalf; ++e) {
                if (kRowsAhead == 2 ? e % 4 == 0 && e < 12 : e % 4 == 0) rows(b, e / 4 + kRowsAhead - 1);
                element(b, e);
              }
              if constexpr (step + 1 == 2 * kHalf) {
                if constexpr (b == 0 && kRowsAhead == 2) rows(1, 0);
                range.fit(d[b], dk, some);
#pragma unroll
                for (int c = 0; c < 2; ++c) w[b][c] = packed<T>(s[b][0], c), x[b][c] = packed<T>(d[b][0], c);
              }
            }
            __builtin_amdgcn_sched_barrier(0);
          });
        }
      }
      if (more) put(now ^ 1u);
      arrived();
    }
  }
  const uint64_t rows_again = __builtin_amdgcn_ballot_w64(some && !(finite<D>(dk) && finite<D>(dv)));
  const uint32_t redo = (uint32_t)rows_again | (uint32_t)(rows_again >> 32);
  if (!some) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) dk[d] = dv[d] = f32x16{};
  }
  const bool mine = span.mine() && !(redo >> (lane & 31u) & 1u);
  float *part_k = p.part + (uint64_t)part * 2u * p.kv_heads * p.rows * D, *part_v = part_k + (uint64_t)p.kv_heads * p.rows * D;
  store_key<T, D>(p, p.grad_k, part_k, kv, j, dk, p.scale / range.by, mine);
  store_key<T, D>(p, p.grad_v, part_v, kv, j, dv, kShift<T> != 0.f ? 0x1p-14f : 1.f, mine);
  for (uint32_t left = redo; left; left &= left - 1u) {
    const uint32_t r = wave * 32u + (uint32_t)__builtin_ctz(left);
    grad_kv_row<T, D>(p, kv, h0, h1, (uint32_t)block.first + r, seen.lo[r], seen.hi[r], part_k, part_v);
  }
}

// Adds the parts' sums in order: a thread 8 elements of a key.  Memory: 8 parts of 8 192 x 2 heads of 128 in 22 us, 6 TB/s.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_attend_join(const Attention p) {
  const uint64_t n = (uint64_t)2 * p.kv_heads * p.rows * (D / 8), of = (uint64_t)blockIdx.x * 256u + threadIdx.x;
  if (of >= n) return;
  const uint32_t piece = (uint32_t)(of % (D / 8));
  if (piece * 8u >= p.size) return;
  const uint64_t key = of / (D / 8), j = key % p.rows, kv = key / p.rows % p.kv_heads;
  float x[8] = {};
  for (uint32_t part = 0; part < p.parts; ++part) {
    const float* from = p.part + (uint64_t)part * 2u * p.kv_heads * p.rows * D + of * 8u;
    const f32x4 a = *(const LMT_GLOBAL f32x4*)from, b = *(const LMT_GLOBAL f32x4*)(from + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += a[e], x[4 + e] += b[e];
  }
  const Heads& to = key / p.rows < p.kv_heads ? p.grad_k : p.grad_v;
  T* row = const_cast<T*>(row_of(head_of<T>(to, (uint32_t)kv), to, (uint32_t)j));
  Vec<T, 8> v;
  v.set(x);
  store_piece(row, piece, v, p.size);
}

// Whether rows of two tensors can go to LDS by themselves: on 16 bytes, and 64 rows within what 32 bits count.
bool direct(const Attention& p, const Heads& a, const Heads& b) {
  const auto fits = [&](const Heads& x) { return ((uintptr_t)x.at & 15u) == 0 && x.row % 8 == 0 && x.head % 8 == 0 && x.row < (1u << 24); };
  return p.size % 8 == 0 && fits(a) && fits(b);
}
template <typename F>
hipError_t with_form(const Attention& p, int dtype, bool straight, F f) {
  const bool plain = p.cap == 0.f && !p.slopes && p.scale > 0.f;
  const auto staged = [&](auto t, auto wide, auto simple) {
    if (straight) return f(t, wide, simple, std::true_type{});
    return f(t, wide, simple, std::false_type{});
  };
  const auto sized = [&](auto t, auto wide) {
    if (plain) return staged(t, wide, std::true_type{});
    return staged(t, wide, std::false_type{});
  };
  const auto typed = [&](auto t) {
    if (p.size <= 64u) return sized(t, std::integral_constant<int, 64>{});
    return sized(t, std::integral_constant<int, 128>{});
  };
  return dtype == LMT_F16 ? typed(_Float16{}) : typed(bf16_t{});
}

}  // namespace

uint32_t attention_parts(uint64_t rows, uint64_t heads, uint64_t kv_heads, uint64_t) {
  // up to four workgroups a compute unit, as long as there are query heads; each part costs 8 bytes an element of k written and read once more
  const uint64_t group = heads / kv_heads, there = ceil_div(rows, kRows) * kv_heads;
  return (uint32_t)std::max<uint64_t>(1, std::min(group, 4 * kCus / there));
}

uint64_t attention_grad_workspace(uint64_t rows, uint64_t heads, uint64_t kv_heads, uint64_t size) {
  const uint64_t parts = attention_parts(rows, heads, kv_heads, size);
  return round_up(4 * rows * heads, 16) + (parts > 1 ? 8 * parts * kv_heads * rows * (size <= 64 ? 64 : 128) : 0);
}

uint64_t attention_launches(uint64_t rows, uint64_t heads) { return ceil_div(rows, kRows) * heads; }

namespace {

// Blocks of the forward pass are cut at the starts of sequences where there are few rounds of them, so that the longest one counts, and sequences are long:
// two blocks of rows on average.  24 causal sequences of up to 1 500, 10 heads: cut 65 us, else 73; but 128 sequences of up to 512, 16 heads: 125 and 118.
// Padded batches start on blocks (16 in 512 rows each: 24 and 22), and the gradient's workgroups gain less than the cuts cost (292 and 280).
uint32_t cuts(const Attention& p) {
  const uint64_t tiles = ceil_div(p.rows, kRows);
  return !p.lengths && p.sequences > 1u && 2ull * p.sequences <= tiles && tiles * p.heads <= 8 * kCus ? p.sequences : 0u;
}

}  // namespace

hipError_t launch_attention(const Attention& q, int dtype, hipStream_t s) {
  Attention p = q;
  p.cuts = cuts(p);
  const uint32_t tiles = (uint32_t)ceil_div(p.rows, kRows) + p.cuts;
  return with_form(p, dtype, direct(p, p.k, p.v), [&](auto t, auto d, auto plain, auto straight) {
    hipLaunchKernelGGL((k_attend<decltype(t), decltype(d)::value, decltype(plain)::value, decltype(straight)::value>), dim3(tiles * p.heads), dim3(kThreads), 0, s, p, tiles);
    return hipGetLastError();
  });
}

hipError_t launch_attention_grad(const Attention& p, int dtype, hipStream_t s) {
  const uint32_t tiles = (uint32_t)ceil_div(p.rows, kRows);
  const hipError_t e = with_form(p, dtype, direct(p, p.k, p.v), [&](auto t, auto d, auto plain, auto straight) {
    hipLaunchKernelGGL((k_attend_grad_q<decltype(t), decltype(d)::value, decltype(plain)::value, decltype(straight)::value>), dim3(tiles * p.heads), dim3(kThreads), 0, s, p, tiles);
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  return with_form(p, dtype, direct(p, p.q, p.grad_out), [&](auto t, auto d, auto plain, auto straight) {
    hipLaunchKernelGGL((k_attend_grad_kv<decltype(t), decltype(d)::value, decltype(plain)::value, decltype(straight)::value>), dim3(tiles * p.kv_heads * p.parts), dim3(kThreads), 0, s, p, tiles);
    if (p.parts > 1u)
      hipLaunchKernelGGL((k_attend_join<decltype(t), decltype(d)::value>), dim3((uint32_t)ceil_div((uint64_t)2 * p.kv_heads * p.rows * (decltype(d)::value / 8), 256)), dim3(256), 0, s, p);
    return hipGetLastError();
  });
}

}  // namespace lmt
