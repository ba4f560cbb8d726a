// Embedding lookup and the gradient of its table (lmt.h).
//
// Lookup: out[t] = scale * table[token[t]].  Every element is read and written once; a row is taken by as many lanes of a
// wavefront as it has pieces, of as many elements as 16 bytes hold of the narrower of the two types, so a wavefront has 64 pieces of a
// long row or several short rows.
//
// Gradient: grad[v] = scale * sum of grad_out[t] over the t with token[t] = v.  The positions t are sorted by token (stable
// radix sort, ten bits at a time at most; up to 16 384 tokens by one workgroup in LDS, while the others clear the table), the sorted
// list is cut into chunks of equal length, and a wavefront sums the rows of one chunk in list order, row after row in
// registers: rows whose tokens lie in one chunk are finished there; a row that goes over a chunk's end is filed as partial
// sums (one in front, one behind per chunk) and joined in chunk order by a last kernel.  Nothing is added atomically: the
// order of every sum depends on the sizes and the tokens alone.
#include "lmt_device.h"
#include "lmt_internal.h"

namespace lmt {
namespace {

constexpr uint32_t kThreads = 256, kWaves = kThreads / 64;

__device__ __forceinline__ uint32_t lane_id() { return threadIdx.x & 63u; }

// ---- lookup ----------------------------------------------------------------------

// Lanes per row: a power of two; rows longer than 64 pieces go in slabs of 64.  Bound by memory: 32 768 rows of 1 024, of 30 522 at random with a
// quarter padding, from fp32 to bf16 in 26 us (29.7 with stores that stay in the L2; bf16 to bf16 18 and 27); 37 rows of 256 in 4.5, a launch.
template <typename TI, typename TO, typename I>
__global__ __launch_bounds__(kThreads) void k_embed(const Embed p, uint32_t lanes_log2, uint32_t slabs, uint64_t n_units) {
  constexpr int V = 16 / (sizeof(TI) > sizeof(TO) ? sizeof(TO) : sizeof(TI));
  const uint32_t lanes = 1u << lanes_log2, per_wave = 64u >> lanes_log2;
  const uint32_t sub = lane_id() >> lanes_log2, at = lane_id() & (lanes - 1u);
  const uint32_t step = gridDim.x * kWaves;
  for (uint64_t unit = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); unit < n_units; unit += step) {
    const uint32_t u = (uint32_t)unit, of_row = u / slabs;  // the output is in memory, so there are fewer than 2^32
    const uint64_t row = (uint64_t)of_row * per_wave + sub;
    const uint32_t col = ((u - of_row * slabs) * 64u + at) * V;
    if (row >= p.n_tokens || col >= p.width) continue;
    const int64_t token = id_at<I>(p.tokens, row);
    const bool there = (uint64_t)token < p.vocab;
    if (!there && p.status && col == 0) atomicOr(p.status, LMT_STATUS_BAD_TOKEN);
    Vec<TI, V> x = {};
    Vec<TO, V> y;
    float f[V];
    const uint32_t n = min((uint32_t)V, p.width - col);
    if (there) {
      const TI* from = static_cast<const TI*>(p.table) + (uint64_t)token * p.table_ld + col;
      if (n == V) load<false>(x, from);
      else load_end(x, from, n, 0.f);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = x.get(i) * p.scale;
    if (!there) {
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = 0.f;
    }
    y.set(f);
    TO* to = static_cast<TO*>(p.out) + row * p.out_ld + col;
    if (n == V) store<true>(to, y);
    else store_end(to, y, n);
  }
}

// ---- sorting the tokens --------------------------------------------------------------

constexpr uint32_t kMaxDigitBits = 10, kMaxBins = 1u << kMaxDigitBits;

// A token's sort key: itself, or `vocab`, behind all others, if it has no gradient.
template <typename I>
__device__ __forceinline__ uint32_t key_of(const EmbedGrad& p, uint32_t t) {
  const int64_t token = id_at<I>(p.tokens, t);
  if (token == p.skip_token) return p.vocab;
  if ((uint64_t)token < p.vocab) return (uint32_t)token;
  if (p.status) atomicOr(p.status, LMT_STATUS_BAD_TOKEN);
  return p.vocab;
}

// Lanes of this wavefront that hold the same digit, among the lanes in `valid`: those that agree bit by bit, four instructions for each.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, uint32_t bits, uint64_t valid) {
  uint32_t lo = (uint32_t)valid, hi = (uint32_t)(valid >> 32);
  for (uint32_t b = 0; b < bits; ++b) {
    const uint32_t mine = (uint32_t)__builtin_amdgcn_sbfe((int)digit, b, 1);  // all ones or zeros
    const uint64_t ones = __ballot(mine != 0);
    lo &= ~((uint32_t)ones ^ mine), hi &= ~((uint32_t)(ones >> 32) ^ mine);
  }
  return (uint64_t)hi << 32 | lo;
}

// Ranks of a wavefront's keys (R x 64 in a row, round by round) among its equal digits; seen[digit], cleared before, counts them.
template <int R>
__device__ __forceinline__ void rank_digits(const uint32_t (&key)[R], uint32_t shift, uint32_t bits, uint32_t n_valid, volatile uint16_t* seen, uint32_t (&rank)[R]) {
  const uint32_t lane = lane_id();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool valid = r * 64u + lane < n_valid;
    const uint32_t digit = key[r] >> shift & ((1u << bits) - 1u);
    const uint64_t same = same_digit(digit, bits, __ballot(valid));
    const uint32_t before = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
    rank[r] = valid ? seen[digit] + before : 0u;
    __builtin_amdgcn_wave_barrier();
    if (valid && before == 0) seen[digit] = (uint16_t)(rank[r] + (uint32_t)__popcll(same));
    __builtin_amdgcn_wave_barrier();
  }
}

// Sum over the threads in front of this one.  sums: LDS, one word per wavefront.
__device__ __forceinline__ uint32_t sum_in_front(uint32_t x, uint32_t* sums) {
  const uint32_t lane = lane_id(), wave = threadIdx.x >> 6;
  uint32_t up_to = x;
#pragma unroll
  for (uint32_t d = 1; d < 64; d *= 2) {
    const uint32_t y = __shfl_up(up_to, d);
    if (lane >= d) up_to += y;
  }
  if (lane == 63) sums[wave] = up_to;
  __syncthreads();
  uint32_t before = up_to - x;
  for (uint32_t w = 0; w < wave; ++w) before += sums[w];
  return before;
}

// Rows of bytes to be cleared, `bytes` of each; a table without gaps is one long row cut into pieces.
struct Clear {
  char* at;
  uint64_t rows, stride, bytes, end;  // end: of the last row
};
__device__ __forceinline__ void clear_rows(const Clear& c, uint64_t first, uint64_t step) {
  for (uint64_t r = first; r < c.rows; r += step) {
    char* row = c.at + r * c.stride;
    const uint64_t n = min(c.bytes, c.end - r * c.stride);
    for (uint64_t b = (uint64_t)lane_id() * 16u; b < n; b += 1024u) {
      if (b + 16u <= n) {
        __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, (LMT_GLOBAL typename At<2>::x4*)(row + b));
      } else {
        for (uint64_t e = b; e < n; e += 2u) *(LMT_GLOBAL uint16_t*)(row + e) = 0;
      }
    }
  }
}

// A token's key and its position.
__device__ __forceinline__ u32x2 pair_at(const u32x2* list, uint64_t i) { return *(const LMT_GLOBAL u32x2*)(list + i); }
__device__ __forceinline__ uint32_t key_at(const u32x2* list, uint64_t i) { return *(const LMT_GLOBAL uint32_t*)(list + i); }

constexpr uint32_t kSortThreads = 1024, kSortWaves = kSortThreads / 64;

// The whole sort of up to 1024 R tokens by workgroup 0, digit after digit in LDS; the other workgroups clear the table
// meanwhile (the rows that get a sum are written twice for that).  The sort is bound by one compute unit's vector issue (an instruction
// stream of about 50 for each 64 tokens and pass): 8 192 tokens of 30 522 in 16.2 us, 600 in 6.0; with the clear of 30 522 x 768 in fp32
// beside it 17.6 (94 MB, 5.3 TB/s; a fill alone reaches 7).
template <typename I, int R>
__global__ __launch_bounds__(kSortThreads) void k_token_sort(const EmbedGrad p, uint32_t passes, uint32_t bits, u32x2* list, const Clear clear) {
  const uint32_t wave = threadIdx.x >> 6, lane = lane_id();
  if (blockIdx.x > 0) {
    clear_rows(clear, (uint64_t)(blockIdx.x - 1u) * kSortWaves + wave, (uint64_t)(gridDim.x - 1u) * kSortWaves);
    return;
  }
  __shared__ uint32_t keys[kSortThreads * R];
  __shared__ uint16_t ats[kSortThreads * R];
  __shared__ uint16_t seen[kSortWaves][kMaxBins];
  __shared__ uint32_t sums[kSortWaves];
  const uint32_t first = wave * (R * 64u), bins = 1u << bits;
  const uint32_t n_valid = p.n_tokens > first ? p.n_tokens - first : 0u;
  uint32_t key[R], at[R], rank[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    at[r] = first + r * 64u + lane;
    key[r] = at[r] < p.n_tokens ? key_of<I>(p, at[r]) : 0u;
  }
  for (uint32_t pass = 0; pass < passes; ++pass) {
    const uint32_t shift = pass * bits;
    for (uint32_t i = threadIdx.x; i < kSortWaves * bins; i += kSortThreads) seen[i >> bits][i & (bins - 1u)] = 0;
    __syncthreads();
    rank_digits<R>(key, shift, bits, n_valid, seen[wave], rank);
    __syncthreads();
    uint32_t count = 0;
    if (threadIdx.x < bins) {
#pragma unroll
      for (uint32_t w = 0; w < kSortWaves; ++w) count += seen[w][threadIdx.x];
    }
    uint32_t to = sum_in_front(count, sums);
    if (threadIdx.x < bins) {
#pragma unroll
      for (uint32_t w = 0; w < kSortWaves; ++w) {
        const uint32_t c = seen[w][threadIdx.x];
        seen[w][threadIdx.x] = (uint16_t)to;
        to += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r * 64u + lane >= n_valid) continue;
      to = seen[wave][key[r] >> shift & (bins - 1u)] + rank[r];
      keys[to] = key[r], ats[to] = (uint16_t)at[r];
    }
    __syncthreads();
    if (pass + 1u == passes) break;
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = keys[first + r * 64u + lane], at[r] = ats[first + r * 64u + lane];
  }
  for (uint32_t i = threadIdx.x; i < p.n_tokens; i += kSortThreads) *(LMT_GLOBAL u32x2*)(list + i) = u32x2{keys[i], ats[i]};
}

// One pass of the sort of more tokens than that: workgroups count their digits, then each adds up the counts and moves its
// tokens.  1024 threads with R tokens each: 2 where that makes up to 256 workgroups, which all read all counts, and 8 above (calls with rows of
// 64, us, 2 and 8: 262 144 tokens 73 and 86, 524 288 110 and 122, 1 048 576 203 and 188).  Bound by latency: 262 144 tokens in two passes of
// 4.7 + 9.6 us (10 MB in and out).  Every workgroup reads the counts of all, so the reading grows with the square of the tokens: nothing beside the rest up to
// a million, 51 us a pass of 4 194 304 tokens (30 522 of them different), 340 of 16 777 216, 8.6 GB; beyond, the form still gives the right order, but a
// sum of the counts in a launch of its own would be the better one.
struct Sort {  // FIRST: from the tokens themselves
  const u32x2* from;
  u32x2* to;
  uint16_t* counts;  // [blocks][bins]
  uint32_t shift, bits, blocks;
};

template <typename I, bool FIRST, int R>
__global__ __launch_bounds__(kSortThreads) void k_token_counts(const EmbedGrad p, const Sort s) {
  __shared__ uint32_t bin[kMaxBins];
  const uint32_t bins = 1u << s.bits;
  uint32_t key[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t t = blockIdx.x * (R * kSortThreads) + r * kSortThreads + threadIdx.x;
    key[r] = t < p.n_tokens ? (FIRST ? key_of<I>(p, t) : key_at(s.from, t)) : ~0u;
  }
  if (threadIdx.x < bins) bin[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (key[r] != ~0u) atomicAdd(&bin[key[r] >> s.shift & (bins - 1u)], 1u);
  __syncthreads();
  if (threadIdx.x < bins) s.counts[(uint64_t)blockIdx.x * bins + threadIdx.x] = (uint16_t)bin[threadIdx.x];
}

template <typename I, bool FIRST, int R>
__global__ __launch_bounds__(kSortThreads) void k_token_move(const EmbedGrad p, const Sort s) {
  __shared__ uint16_t seen[kSortWaves][kMaxBins];  // of a wavefront's tokens so far
  __shared__ uint32_t start[kMaxBins];             // where this workgroup's tokens of a digit go
  __shared__ uint32_t all_part[8 * kSortThreads], front_part[8 * kSortThreads];
  __shared__ uint32_t sums[kSortWaves];
  const uint32_t bins = 1u << s.bits, wave = threadIdx.x >> 6, lane = lane_id();
  const uint32_t first = blockIdx.x * (R * kSortThreads) + wave * (R * 64u);
  const uint32_t n_valid = p.n_tokens > first ? p.n_tokens - first : 0u;
  uint32_t key[R], at[R], rank[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t t = first + r * 64u + lane;
    key[r] = 0, at[r] = t;
    if (t < p.n_tokens) {
      if (FIRST) {
        key[r] = key_of<I>(p, t);
      } else {
        const u32x2 x = pair_at(s.from, t);
        key[r] = x.x, at[r] = x.y;
      }
    }
  }
  for (uint32_t i = threadIdx.x; i < kSortWaves * bins; i += kSortThreads) seen[i >> s.bits][i & (bins - 1u)] = 0;
  // the counts of all workgroups and of those in front: a thread has eight digits of every n-th workgroup
  {
    const uint32_t across = bins / 8u, groups = kSortThreads / across, group = threadIdx.x / across, d = threadIdx.x % across * 8u;
    uint32_t all[8] = {}, front[8] = {};
#pragma unroll 4
    for (uint32_t b = group; b < s.blocks; b += groups) {
      const u32x4 w = *(const LMT_GLOBAL u32x4*)(s.counts + (uint64_t)b * bins + d);
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t c = w[i / 2] >> (16 * (i & 1)) & 0xffffu;
        all[i] += c;
        front[i] += b < blockIdx.x ? c : 0u;
      }
    }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) all_part[group * bins + d + i] = all[i], front_part[group * bins + d + i] = front[i];
  }
  __syncthreads();
  rank_digits<R>(key, s.shift, s.bits, n_valid, seen[wave], rank);
  // where this workgroup's tokens of a digit go: behind the smaller digits of all workgroups and this digit of those in front
  uint32_t all = 0, front = 0;
  if (threadIdx.x < bins)
    for (uint32_t g = threadIdx.x; g < 8u * kSortThreads; g += bins) all += all_part[g], front += front_part[g];
  const uint32_t before = sum_in_front(all, sums);  // a barrier for `seen` too
  if (threadIdx.x < bins) {
    start[threadIdx.x] = before + front;
    uint32_t to = 0;
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) {
      const uint32_t c = seen[w][threadIdx.x];
      seen[w][threadIdx.x] = (uint16_t)to;
      to += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r * 64u + lane >= n_valid) continue;
    const uint32_t d = key[r] >> s.shift & (bins - 1u);
    *(LMT_GLOBAL u32x2*)(s.to + start[d] + seen[wave][d] + rank[r]) = u32x2{key[r], at[r]};
  }
}

// ---- summing the rows ------------------------------------------------------------------

struct Sums {
  const u32x2* list;  // sorted: token and position
  float* partial;      // [2][chunks][pieces][V]: a chunk's share of the row that comes over its start; of the one that leaves over its end
  uint32_t chunk, n_chunks, pieces;
};

// First index in [lo, hi) of the sorted list whose key is not below `key`.
__device__ __forceinline__ uint32_t lower_bound(const u32x2* list, uint32_t lo, uint32_t hi, uint32_t key) {
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2u;
    if (key_at(list, mid) < key) lo = mid + 1u;
    else hi = mid;
  }
  return lo;
}

// Row `i` of a matrix with rows of ld elements, `offset` bytes (32 bits, a lane's) into it: for a uniform i the row's address stays in
// scalar registers, where computing it costs the vector unit nothing.
template <typename T>
__device__ __forceinline__ T* in_row(const void* base, uint32_t i, uint64_t ld, uint32_t offset) {
  return (T*)((LMT_GLOBAL char*)base + i * (ld * sizeof(T)) + offset);
}

// A lane's V columns of a row: V at a time, the last ones from the end (width >= V), so that every load is a whole vector; of those only
// the ones from `own` on are the lane's to write (V: none).
template <int V>
struct Piece {
  uint32_t index, col, own;
  __device__ __forceinline__ Piece(uint32_t i, uint32_t width, uint32_t pieces) {
    index = min(i, pieces - 1u);
    col = min(index * V, width - V);
    own = i < pieces ? index * V - col : (uint32_t)V;
  }
};
template <typename T, int V>
__device__ __forceinline__ void store_own(T* to, const Vec<T, V>& y, uint32_t own) {
  if (own == 0) {
    store<true>(to, y);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if ((uint32_t)i >= own) store1(to + i, from_f32<T>(y.get(i)));
  }
}
template <typename TO, int V>
__device__ __forceinline__ void put_row(const EmbedGrad& p, uint32_t key, const Piece<V>& piece, const float (&sum)[V], const Vec<TO, V>& old, bool add) {
  float f[V];
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = add ? __builtin_fmaf(sum[i], p.scale, old.get(i)) : sum[i] * p.scale;
  Vec<TO, V> y;
  y.set(f);
  store_own(in_row<TO>(p.grad, key, p.grad_ld, piece.col * (uint32_t)sizeof(TO)), y, piece.own);
}
template <int V>
__device__ __forceinline__ float* partial_at(const Sums& s, uint32_t c, const Piece<V>& piece) {  // c: of the chunk, plus n_chunks for its end
  return s.partial + ((uint64_t)c * s.pieces + piece.index) * V;
}

// A wavefront loads rows in batches, one ahead of the one that it adds, and with them, when it accumulates (ADD), what the table
// holds for the tokens that end there.
// Workgroups [0, sum_blocks): a wavefront per chunk and slab of 64 pieces.  Behind them, where the table has not been cleared: rows
// of tokens that do not occur, 64 per wavefront, are.  Bound by memory: 262 144 rows of 1 024 in bf16, a quarter of them padding, added to a
// table of 30 522 in fp32, 130 us (575 MB with the table's rows that occur, in and out, 4.4 TB/s); 8 192 rows of 768, 7.5 us.
template <typename TI, typename TO, int V, bool ADD>
__global__ __launch_bounds__(kThreads) void k_token_sums(const EmbedGrad p, const Sums s, uint32_t slabs, uint32_t sum_blocks) {
  constexpr uint32_t kBatch = ADD ? 4 : 8;
  const uint32_t lane = lane_id();
  if (!ADD && blockIdx.x >= sum_blocks) {
    const uint64_t v0 = ((uint64_t)(blockIdx.x - sum_blocks) * kWaves + (threadIdx.x >> 6)) * 64u;
    bool absent = false;
    if (v0 + lane < p.vocab) {
      const uint32_t i = lower_bound(s.list, 0, p.n_tokens, (uint32_t)v0 + lane);
      absent = i == p.n_tokens || key_at(s.list, i) != (uint32_t)v0 + lane;
    }
    for (uint64_t rows = __ballot(absent); rows != 0; rows &= rows - 1ull) {
      TO* row = static_cast<TO*>(p.grad) + (v0 + (uint64_t)(__ffsll((unsigned long long)rows) - 1)) * p.grad_ld;
      for (uint32_t q = lane; q < s.pieces; q += 64u) {
        const Piece<V> piece(q, p.width, s.pieces);
        Vec<TO, V> zero;
        const float f[V] = {};
        zero.set(f);
        store_own(row + piece.col, zero, piece.own);
      }
    }
    return;
  }
  const uint32_t unit = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t c = unit / slabs;
  if (c >= s.n_chunks) return;
  const Piece<V> piece(unit % slabs * 64u + lane, p.width, s.pieces);
  const uint32_t lo = c * s.chunk, hi = min(p.n_tokens, lo + s.chunk);
  const uint32_t before = __builtin_amdgcn_readfirstlane(lo > 0 ? key_at(s.list, lo - 1u) : ~0u);
  const uint32_t behind = __builtin_amdgcn_readfirstlane(hi < p.n_tokens ? key_at(s.list, hi) : ~0u);
  float sum[V];
  uint32_t run = ~0u;       // the token whose rows are being summed
  bool from_front = false;  // ... since the chunk in front
  struct Batch {
    Vec<TI, V> x[kBatch];
    Vec<TO, V> old[ADD ? kBatch : 1];
  };
  for (uint32_t i0 = lo; i0 < hi; i0 += 64u) {
    const uint32_t i = min(i0 + lane, hi - 1u);
    const u32x2 pair = pair_at(s.list, i);
    const uint32_t next = i + 1u < hi ? key_at(s.list, i + 1u) : ~0u;
    const uint64_t valid = __ballot(i0 + lane < hi && pair.x < p.vocab);  // those without gradient are last
    const uint64_t ends = __ballot(pair.x != next) & valid;
    const uint32_t count = (uint32_t)__popcll(valid);
    if (count == 0) break;
    const auto fetch = [&](Batch& b, uint32_t j0) {
#pragma unroll
      for (uint32_t j = 0; j < kBatch; ++j) {
        const uint32_t at = min(j0 + j, count - 1u);
        load<true>(b.x[j], in_row<const TI>(p.grad_out, __builtin_amdgcn_readlane(pair.y, at), p.grad_out_ld, piece.col * (uint32_t)sizeof(TI)));
        if constexpr (ADD) {
          if (ends >> at & 1ull) load<true>(b.old[j], in_row<const TO>(p.grad, __builtin_amdgcn_readlane(pair.x, at), p.grad_ld, piece.col * (uint32_t)sizeof(TO)));
        }
      }
    };
    const auto add = [&](const Batch& b, uint32_t j0) {
#pragma unroll
      for (uint32_t j = 0; j < kBatch; ++j) {
        if (j0 + j >= count) break;
        const uint32_t k = __builtin_amdgcn_readlane(pair.x, j0 + j);
        if (k != run) {
          run = k, from_front = i0 + j0 + j == lo && k == before;
#pragma unroll
          for (int v = 0; v < V; ++v) sum[v] = 0.f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += b.x[j].get(v);
        if (ends >> (j0 + j) & 1ull) {
          if (from_front || (i0 + j0 + j + 1u == hi && k == behind)) {
            float* to = partial_at(s, from_front ? c : s.n_chunks + c, piece);
#pragma unroll
            for (int v = 0; v < V; ++v) *(LMT_GLOBAL float*)(to + v) = sum[v];
          } else {
            put_row<TO, V>(p, k, piece, sum, b.old[ADD ? j : 0], ADD);
          }
        }
      }
    };
    Batch a, b;
    fetch(a, 0);
    for (uint32_t j0 = 0; j0 < count; j0 += 2u * kBatch) {
      fetch(b, j0 + kBatch);
      add(a, j0);
      fetch(a, j0 + 2u * kBatch);
      add(b, j0 + kBatch);
    }
    if (count < 64u) break;
  }
}

// Rows that go over chunk ends.  A wavefront looks at one chunk and, if such a row starts there, adds its partial sums; a row of over
// kLong chunks is left to all wavefronts of the workgroup, which add every sixteenth of its chunks, then the sixteen sums in order.
// Bound by the latency of a chain of dependent reads (list, bounds, sums): 5 us after 8 192 tokens, 6 after 262 144.
constexpr uint32_t kJoinWaves = 16, kLong = 16;
template <typename TO, int V>
__global__ __launch_bounds__(64 * kJoinWaves) void k_token_joins(const EmbedGrad p, const Sums s) {
  __shared__ float part[kJoinWaves][V][64];
  __shared__ uint32_t long_last[kJoinWaves];
  const uint32_t lane = lane_id(), wave = threadIdx.x >> 6;
  const Piece<V> piece(blockIdx.y * 64u + lane, p.width, s.pieces);
  const auto get = [&](uint32_t c, float (&x)[V]) {
    const float* from = partial_at(s, c, piece);
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = *(const LMT_GLOBAL float*)(from + v);
  };
  // adds chunks d, d + step, ... up to the last one, eight loads ahead
  const auto add = [&](float (&sum)[V], uint32_t d, uint32_t last, uint32_t step) {
    for (; d <= last; d += 8u * step) {
      float x[8][V];
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) get(min(d + i * step, last), x[i]);
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += d + i * step <= last ? x[i][v] : 0.f;
    }
  };
  const auto old_of = [&](uint32_t key, Vec<TO, V>& old) {
    if (p.accumulate) load<true>(old, static_cast<const TO*>(p.grad) + (uint64_t)key * p.grad_ld + piece.col);
  };
  const uint32_t c = blockIdx.x * kJoinWaves + wave;
  uint32_t last = 0, key = 0;
  if (c + 1u < s.n_chunks) {
    const uint32_t lo = c * s.chunk, hi = lo + s.chunk;
    key = key_at(s.list, hi - 1u);
    const uint32_t next = key_at(s.list, hi), start = key_at(s.list, lo), before = lo > 0 ? key_at(s.list, lo - 1u) : ~0u;
    if (key < p.vocab && next == key && !(start == key && before == key)) {  // a row leaves that has not come over the start
      last = c;
      for (uint64_t more = ~0ull; more == ~0ull; last += more == ~0ull ? 64u : (uint32_t)__ffsll((unsigned long long)~more) - 1u)
        more = __ballot((uint64_t)last + 1u + lane < s.n_chunks && key_at(s.list, (uint64_t)(last + 1u + lane) * s.chunk) == key);
    }
  }
  const bool is_long = last > c + kLong;
  if (last != 0 && !is_long) {
    float sum[V];
    Vec<TO, V> old;
    old_of(key, old);
    get(s.n_chunks + c, sum);
    add(sum, c + 1u, last, 1u);
    put_row<TO, V>(p, key, piece, sum, old, p.accumulate);
  }
  if (lane == 0) long_last[wave] = is_long ? last : 0u;
  __syncthreads();
  for (uint32_t w = 0; w < kJoinWaves; ++w) {
    last = long_last[w];
    if (last == 0) continue;
    const uint32_t cw = blockIdx.x * kJoinWaves + w;
    float sum[V] = {};
    Vec<TO, V> old;
    if (wave == 0) {
      key = key_at(s.list, (uint64_t)last * s.chunk);
      old_of(key, old);
      get(s.n_chunks + cw, sum);
    }
    add(sum, cw + 1u + wave, last, kJoinWaves);
#pragma unroll
    for (int v = 0; v < V; ++v) part[wave][v][lane] = sum[v];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (uint32_t x = 1; x < kJoinWaves; ++x)
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += part[x][v][lane];
      put_row<TO, V>(p, key, piece, sum, old, p.accumulate);
    }
    __syncthreads();
  }
}

// A table without a token: zeros.
template <typename TO>
__global__ __launch_bounds__(kThreads) void k_token_none(const EmbedGrad p) {
  for (uint64_t row = blockIdx.x; row < p.vocab; row += gridDim.x)
    for (uint32_t col = threadIdx.x; col < p.width; col += kThreads)
      store1(static_cast<TO*>(p.grad) + row * p.grad_ld + col, from_f32<TO>(0.f));
}

// ---- launches ------------------------------------------------------------------------

// Positions per chunk.  Few tokens: short ones, so that more wavefronts load (us with 4, 8, 16: 600 tokens 14.2, 14.6, 16.1; 2 048 into a
// table of 30 522 x 768 with 8, 16: 26.1, 27.1; 8 192: 31.4, 30.1, the joins cost more).  Many: about a thousand chunks (262 144 tokens with rows of 1 024
// 139 us, with two thousand 141, with four 145).  Drawn for rows of 1 024, four wavefronts a chunk; rows of up to 256 have one, and 1 024 wavefronts do not fill the
// card: 262 144 tokens with rows of 64, 128 and 256 in bf16 all take 74 to 80 us where 1 024 take 191, and 16 777 216 with rows of 64 spend 2 000 of
// 2 750 in the sums, 1.1 TB/s.  Shorter chunks for narrow rows have not been measured.
uint32_t chunk_of(uint64_t n_tokens) {
  uint64_t chunk = n_tokens <= 1024 ? 4 : n_tokens <= 4096 ? 8 : 16;
  while (chunk * 1024u < n_tokens) chunk *= 2;
  return (uint32_t)chunk;
}

// Tokens that one workgroup sorts.  A whole call into 30 522 x 768, with more than 2 048 tokens sorted by many workgroups instead: 4 096 tokens
// 28 us (56), 8 192 30 (56), 16 384 47 (64); adding to the table, where nothing has to be cleared meanwhile, 23 (33), 32 (37), 51 (46).  One border for both,
// since the workspace is asked for without the flag: it costs the upper end of what is added a tenth.
constexpr uint64_t kMostSorted = 16 * kSortThreads;

struct Passes {
  uint32_t n, bits, rounds, blocks;
};
Passes passes_of(uint64_t n_tokens, uint64_t vocab) {
  uint32_t bits = 1;
  while (vocab >> bits) ++bits;  // keys 0 .. vocab
  const uint32_t n = (uint32_t)ceil_div(bits, kMaxDigitBits);
  const uint32_t rounds = n_tokens <= 256u * 2u * kSortThreads ? 2u : 8u;
  return {n, std::max(3u, (uint32_t)ceil_div(bits, n)), rounds, (uint32_t)ceil_div(n_tokens, rounds * kSortThreads)};
}

struct Parts {  // offsets in bytes
  uint64_t list[2], counts, partial, total;
};
Parts parts_of(uint64_t n_tokens, uint64_t vocab, uint64_t width) {
  const Passes passes = passes_of(n_tokens, vocab);
  const uint64_t list = round_up(8 * n_tokens, 256), rows = 4 * round_up(width, 8) * ceil_div(n_tokens, chunk_of(n_tokens));
  const bool small = n_tokens <= kMostSorted;
  Parts w{};
  w.list[0] = 0, w.list[1] = list;
  w.counts = 2 * list;
  w.partial = small ? list : w.counts + round_up(2 * (uint64_t)passes.blocks << passes.bits, 256);
  w.total = w.partial + 2 * rows;
  return w;
}

template <int N>
struct Const {
  static constexpr int value = N;
};
template <typename F>
hipError_t with_float(int dtype, F f) {
  switch (dtype) {
    case LMT_F32: return f(float{});
    case LMT_F16: return f(_Float16{});
    default: return f(bf16_t{});
  }
}
template <typename F>
hipError_t with_id(int dtype, F f) {
  return dtype == LMT_I64 ? f(int64_t{}) : f(int32_t{});
}

}  // namespace

hipError_t launch_embed(const Embed& p, int table_dtype, int token_dtype, int out_dtype, hipStream_t s) {
  const uint32_t v = table_dtype == LMT_F32 && out_dtype == LMT_F32 ? 4u : 8u;
  const uint32_t pieces = (p.width + v - 1u) / v;
  uint32_t lanes_log2 = 0;
  while (lanes_log2 < 6u && (1u << lanes_log2) < pieces) ++lanes_log2;
  const uint32_t slabs = (uint32_t)ceil_div(pieces, 64u);
  const uint64_t units = ceil_div(p.n_tokens, 64u >> lanes_log2) * slabs;
  const uint32_t grid = (uint32_t)std::min<uint64_t>(ceil_div(units, kWaves), 1u << 20);
  return with_float(table_dtype, [&](auto ti) {
    return with_float(out_dtype, [&](auto to) {
      return with_id(token_dtype, [&](auto id) {
        hipLaunchKernelGGL((k_embed<decltype(ti), decltype(to), decltype(id)>), dim3(grid), dim3(kThreads), 0, s, p, lanes_log2, slabs, units);
        return hipGetLastError();
      });
    });
  });
}

uint64_t embed_grad_workspace(uint64_t n_tokens, uint64_t vocab, uint64_t width) {
  if (n_tokens == 0 || vocab == 0 || width == 0) return 0;
  return parts_of(n_tokens, vocab, width).total;
}

hipError_t launch_embed_grad(const EmbedGrad& p, int grad_out_dtype, int token_dtype, int grad_dtype, void* workspace, hipStream_t s) {
  if (p.n_tokens == 0) {
    return with_float(grad_dtype, [&](auto to) {
      hipLaunchKernelGGL((k_token_none<decltype(to)>), dim3(std::min(p.vocab, 1u << 16)), dim3(kThreads), 0, s, p);
      return hipGetLastError();
    });
  }
  const Passes passes = passes_of(p.n_tokens, p.vocab);
  const Parts w = parts_of(p.n_tokens, p.vocab, p.width);
  char* base = static_cast<char*>(workspace);
  u32x2* list[2] = {(u32x2*)(base + w.list[0]), (u32x2*)(base + w.list[1])};
  const bool small = p.n_tokens <= kMostSorted, cleared = small && !p.accumulate;
  uint32_t last = 0;
  hipError_t e;
  if (small) {
    const uint64_t size = grad_dtype == LMT_F32 ? 4 : 2, bytes = p.width * size, stride = p.grad_ld * size, end = (p.vocab - 1) * stride + bytes;
    const Clear clear = p.grad_ld == p.width ? Clear{static_cast<char*>(p.grad), ceil_div(end, 4096), 4096, 4096, end} : Clear{static_cast<char*>(p.grad), p.vocab, stride, bytes, end};
    const uint32_t grid = 1u + (p.accumulate ? 0u : (uint32_t)std::min<uint64_t>(8 * kCus - 1u, ceil_div(clear.rows, kSortWaves)));
    e = with_id(token_dtype, [&](auto id) {
      typedef decltype(id) I;
      const auto kernel = p.n_tokens <= 2 * kSortThreads ? k_token_sort<I, 2> : p.n_tokens <= 4 * kSortThreads ? k_token_sort<I, 4> : p.n_tokens <= 8 * kSortThreads ? k_token_sort<I, 8> : k_token_sort<I, 16>;
      hipLaunchKernelGGL(kernel, dim3(grid), dim3(kSortThreads), 0, s, p, passes.n, passes.bits, list[0], clear);
      return hipGetLastError();
    });
  } else {
    last = (passes.n - 1) & 1;
    e = with_id(token_dtype, [&](auto id) {
      typedef decltype(id) I;
      for (uint32_t i = 0; i < passes.n; ++i) {
        const Sort sort{list[(i + 1) & 1], list[i & 1], (uint16_t*)(base + w.counts), i * passes.bits, passes.bits, passes.blocks};
        const bool few = passes.rounds == 2;
        hipLaunchKernelGGL((i == 0 ? few ? k_token_counts<I, true, 2> : k_token_counts<I, true, 8> : few ? k_token_counts<I, false, 2> : k_token_counts<I, false, 8>),
                           dim3(passes.blocks), dim3(kSortThreads), 0, s, p, sort);
        hipLaunchKernelGGL((i == 0 ? few ? k_token_move<I, true, 2> : k_token_move<I, true, 8> : few ? k_token_move<I, false, 2> : k_token_move<I, false, 8>),
                           dim3(passes.blocks), dim3(kSortThreads), 0, s, p, sort);
      }
      return hipGetLastError();
    });
  }
  if (e != hipSuccess) return e;
  const uint32_t chunk = chunk_of(p.n_tokens), n_chunks = (uint32_t)ceil_div(p.n_tokens, chunk);
  return with_float(grad_out_dtype, [&](auto ti) {
    return with_float(grad_dtype, [&](auto to) {
      typedef decltype(ti) TI;
      typedef decltype(to) TO;
      const auto go = [&](auto n) {
        constexpr int V = decltype(n)::value;
        const Sums sums{list[last], (float*)(base + w.partial), chunk, n_chunks, (uint32_t)ceil_div(p.width, V)};
        const uint32_t slabs = (uint32_t)ceil_div(sums.pieces, 64);
        const uint32_t sum_blocks = (uint32_t)ceil_div((uint64_t)n_chunks * slabs, kWaves);
        const uint32_t clear_blocks = p.accumulate || cleared ? 0u : (uint32_t)ceil_div(p.vocab, 64u * kWaves);
        hipLaunchKernelGGL((p.accumulate ? k_token_sums<TI, TO, V, true> : k_token_sums<TI, TO, V, false>), dim3(sum_blocks + clear_blocks), dim3(kThreads), 0, s, p, sums, slabs, sum_blocks);
        if (n_chunks > 1)
          hipLaunchKernelGGL((k_token_joins<TO, V>), dim3((uint32_t)ceil_div(n_chunks - 1u, kJoinWaves), slabs), dim3(64 * kJoinWaves), 0, s, p, sums);
        return hipGetLastError();
      };
      constexpr int V = 4;
      return p.width >= (uint32_t)V ? go(Const<V>{}) : go(Const<1>{});
    });
  });
}

}  // namespace lmt
