// Embedding lookup and the gradient of its table (lmt.h).
//
// Lookup: out[t] = scale * table[token[t]].  Every element is read and written once; a row is taken by as many lanes of a
// wavefront as it has pieces of 16 bytes (of the wider type's elements), so a wavefront has one piece of a long row or several
// short rows.
//
// Gradient: grad[v] = scale * sum of grad_out[t] over the t with token[t] = v.  The positions t are sorted by token (stable
// radix sort, ten bits at a time at most), the sorted list is cut into chunks of equal length, and a wavefront sums the
// rows of one chunk in list order, row after row in registers: rows whose tokens lie in one chunk are finished there; a
// row that goes over a chunk's end is filed as partial sums (one in front, one behind per chunk) and joined in chunk order by a
// last kernel.  Nothing is added atomically: the order of every sum depends on the sizes and the tokens alone.
#include "lmt_device.h"
#include "lmt_internal.h"

namespace lmt {
namespace {

constexpr uint32_t kThreads = 256, kWaves = kThreads / 64;

__device__ __forceinline__ uint32_t lane_id() { return threadIdx.x & 63u; }

// ---- lookup ----------------------------------------------------------------------

// Lanes per row: a power of two; rows longer than 64 pieces go in slabs of 64.
template <typename TI, typename TO, typename I>
__global__ __launch_bounds__(kThreads) void k_embed(const Embed p, uint32_t lanes_log2, uint32_t slabs, uint64_t n_units) {
  constexpr int V = 16 / (sizeof(TI) > sizeof(TO) ? sizeof(TO) : sizeof(TI));
  const uint32_t lanes = 1u << lanes_log2, per_wave = 64u >> lanes_log2;
  const uint32_t sub = lane_id() >> lanes_log2, at = lane_id() & (lanes - 1u);
  const uint64_t step = (uint64_t)gridDim.x * kWaves;
  for (uint64_t u = (uint64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); u < n_units; u += step) {
    const uint64_t row = u / slabs * per_wave + sub;
    const uint32_t col = ((uint32_t)(u % slabs) * 64u + at) * V;
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
    if (n == V) store<false>(to, y);
    else store_end(to, y, n);
  }
}

// ---- sorting the tokens --------------------------------------------------------------

constexpr uint32_t kMaxDigitBits = 10, kMaxBins = 1u << kMaxDigitBits;
constexpr uint32_t kRounds = 16, kSortBlock = kThreads * kRounds;  // tokens a workgroup counts and moves

// A token's sort key: itself, or `vocab`, behind all others, if it has no gradient.
template <typename I>
__device__ __forceinline__ uint32_t key_of(const EmbedGrad& p, uint32_t t) {
  const int64_t token = id_at<I>(p.tokens, t);
  if (token == p.skip_token) return p.vocab;
  if ((uint64_t)token < p.vocab) return (uint32_t)token;
  if (p.status) atomicOr(p.status, LMT_STATUS_BAD_TOKEN);
  return p.vocab;
}

struct Sort {  // one pass of the radix sort: keys and positions from, keys and positions to (FIRST: from the tokens themselves)
  const uint32_t *key, *at;
  uint32_t *key_to, *at_to;
  uint32_t* counts;  // [blocks][bins]
  uint32_t shift, bits;
};

template <typename I, bool FIRST>
__global__ __launch_bounds__(kThreads) void k_token_counts(const EmbedGrad p, const Sort s) {
  __shared__ uint32_t bin[kMaxBins];
  const uint32_t bins = 1u << s.bits;
  for (uint32_t i = threadIdx.x; i < bins; i += kThreads) bin[i] = 0;
  __syncthreads();
#pragma unroll 4
  for (uint32_t r = 0; r < kRounds; ++r) {
    const uint32_t t = blockIdx.x * kSortBlock + r * kThreads + threadIdx.x;
    if (t < p.n_tokens) {
      const uint32_t key = FIRST ? key_of<I>(p, t) : s.key[t];
      atomicAdd(&bin[key >> s.shift & (bins - 1u)], 1u);
    }
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < bins; i += kThreads) s.counts[(uint64_t)blockIdx.x * bins + i] = bin[i];
}

// Lanes of this wavefront that hold the same digit, among the lanes in `valid`.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, uint32_t bits, uint64_t valid) {
  uint64_t same = valid;
  for (uint32_t b = 0; b < bits; ++b) {
    const bool one = digit >> b & 1u;
    const uint64_t ones = __ballot(one);
    same &= one ? ones : ~ones;
  }
  return same;
}

template <typename I, bool FIRST>
__global__ __launch_bounds__(kThreads) void k_token_move(const EmbedGrad p, const Sort s, uint32_t n_blocks) {
  __shared__ uint32_t seen[kWaves][kMaxBins];  // per wavefront: how many of a digit so far; then where its next one goes
  __shared__ uint32_t wave_sum[kWaves];
  const uint32_t bins = 1u << s.bits, wave = threadIdx.x >> 6, lane = lane_id();
  for (uint32_t i = threadIdx.x; i < kWaves * kMaxBins; i += kThreads) seen[i / kMaxBins][i % kMaxBins] = 0;
  __syncthreads();
  // ranks among the wavefront's equal digits; a wavefront has 16 x 64 consecutive positions
  uint32_t key[kRounds], at[kRounds], rank[kRounds];
  volatile uint32_t* mine = seen[wave];
  const uint32_t first = blockIdx.x * kSortBlock + wave * (kRounds * 64u);
#pragma unroll
  for (uint32_t r = 0; r < kRounds; ++r) {
    const uint32_t t = first + r * 64u + lane;
    key[r] = 0, at[r] = t;
    if (t < p.n_tokens) {
      key[r] = FIRST ? key_of<I>(p, t) : s.key[t];
      if (!FIRST) at[r] = s.at[t];
    }
  }
#pragma unroll
  for (uint32_t r = 0; r < kRounds; ++r) {
    const bool valid = first + r * 64u + lane < p.n_tokens;
    const uint32_t digit = key[r] >> s.shift & (bins - 1u);
    const uint64_t same = same_digit(digit, s.bits, __ballot(valid));
    const uint32_t before = (uint32_t)__popcll(same & ((1ull << lane) - 1ull));
    rank[r] = 0;
    if (valid) rank[r] = mine[digit] + before;
    __builtin_amdgcn_wave_barrier();
    if (valid && before == 0) mine[digit] = rank[r] + (uint32_t)__popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  // where each digit of this workgroup starts: the smaller digits of all workgroups, this digit of the workgroups in front
  uint32_t in_front[kMaxBins / kThreads], sum = 0;
  const uint32_t per = (bins + kThreads - 1u) / kThreads;  // digits threadIdx.x * per ...
#pragma unroll
  for (uint32_t j = 0; j < kMaxBins / kThreads; ++j) {
    const uint32_t d = threadIdx.x * per + j;
    in_front[j] = 0;
    if (j >= per || d >= bins) continue;
    uint32_t all = 0;
    for (uint32_t b = 0; b < n_blocks; ++b) {
      const uint32_t c = s.counts[(uint64_t)b * bins + d];
      if (b < blockIdx.x) in_front[j] += c;
      all += c;
    }
    in_front[j] += sum;
    sum += all;
  }
  uint32_t before = sum;  // exclusive sum over the threads
#pragma unroll
  for (uint32_t d = 1; d < 64; d *= 2) {
    const uint32_t x = __shfl_up(before, d);
    if (lane >= d) before += x;
  }
  if (lane == 63) wave_sum[wave] = before;
  before -= sum;
  __syncthreads();
  for (uint32_t w = 0; w < wave; ++w) before += wave_sum[w];
#pragma unroll
  for (uint32_t j = 0; j < kMaxBins / kThreads; ++j) {
    const uint32_t d = threadIdx.x * per + j;
    if (j >= per || d >= bins) continue;
    uint32_t to = before + in_front[j];
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) {
      const uint32_t c = seen[w][d];
      seen[w][d] = to;
      to += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (uint32_t r = 0; r < kRounds; ++r) {
    if (first + r * 64u + lane >= p.n_tokens) continue;
    const uint32_t to = seen[wave][key[r] >> s.shift & (bins - 1u)] + rank[r];
    s.key_to[to] = key[r];
    s.at_to[to] = at[r];
  }
}

// ---- summing the rows ------------------------------------------------------------------

struct Sums {
  const uint32_t *key, *at;  // sorted: token and position
  float *front, *behind;     // [chunks][width]: a chunk's share of the row that comes over its start, of the row that leaves over its end
  uint32_t chunk, n_chunks;
};

// First index in [lo, hi) of the sorted keys that is not below `key`.
__device__ __forceinline__ uint32_t lower_bound(const uint32_t* keys, uint32_t lo, uint32_t hi, uint32_t key) {
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2u;
    if (keys[mid] < key) lo = mid + 1u;
    else hi = mid;
  }
  return lo;
}

// V elements of fp32 of a workspace row whose length may be odd.
template <int V>
__device__ __forceinline__ void put_partial(float* to, const float (&x)[V], uint32_t n) {
#pragma unroll
  for (int i = 0; i < V; ++i)
    if ((uint32_t)i < n) store1(to + i, x[i]);
}

template <typename TO, int V>
__device__ __forceinline__ void put_row(const EmbedGrad& p, uint32_t key, uint32_t col, uint32_t n, const float (&sum)[V]) {
  TO* to = static_cast<TO*>(p.grad) + (uint64_t)key * p.grad_ld + col;
  Vec<TO, V> y = {};
  float f[V];
  if (p.accumulate) {
    if (n == V) load<false>(y, to);
    else load_end(y, to, n, 0.f);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = p.accumulate ? __builtin_fmaf(sum[i], p.scale, y.get(i)) : sum[i] * p.scale;
  y.set(f);
  if (n == V) store<false>(to, y);
  else store_end(to, y, n);
}

constexpr uint32_t kBatch = 8;  // rows in flight per wavefront

// Workgroups [0, sum_blocks): a wavefront per chunk and slab of 64 pieces.  Behind them, without LMT_ACCUMULATE: rows of tokens that
// do not occur, 64 per wavefront, are cleared.
template <typename TI, typename TO>
__global__ __launch_bounds__(kThreads) void k_token_sums(const EmbedGrad p, const Sums s, uint32_t slabs, uint32_t sum_blocks) {
  constexpr int V = 16 / sizeof(TI);
  const uint32_t lane = lane_id();
  if (blockIdx.x >= sum_blocks) {
    const uint64_t v0 = ((uint64_t)(blockIdx.x - sum_blocks) * kWaves + (threadIdx.x >> 6)) * 64u;
    bool absent = false;
    if (v0 + lane < p.vocab) {
      const uint32_t i = lower_bound(s.key, 0, p.n_tokens, (uint32_t)v0 + lane);
      absent = i == p.n_tokens || s.key[i] != (uint32_t)v0 + lane;
    }
    constexpr int Z = 16 / sizeof(TO);
    for (uint64_t rows = __ballot(absent); rows != 0; rows &= rows - 1ull) {
      TO* row = static_cast<TO*>(p.grad) + (v0 + (uint64_t)(__ffsll((unsigned long long)rows) - 1)) * p.grad_ld;
      for (uint32_t col = lane * Z; col < p.width; col += 64u * Z) {
        const Vec<TO, Z> zero = {};
        const uint32_t n = min((uint32_t)Z, p.width - col);
        if (n == Z) store<false>(row + col, zero);
        else store_end(row + col, zero, n);
      }
    }
    return;
  }
  const uint32_t unit = blockIdx.x * kWaves + (threadIdx.x >> 6);
  const uint32_t c = unit / slabs;
  if (c >= s.n_chunks) return;
  const uint32_t col = (unit % slabs * 64u + lane) * V;
  const uint32_t n = col < p.width ? min((uint32_t)V, p.width - col) : 0u;
  const uint32_t lo = c * s.chunk, hi = min(p.n_tokens, lo + s.chunk);
  const uint32_t before = lo > 0 ? s.key[lo - 1u] : ~0u, behind = hi < p.n_tokens ? s.key[hi] : ~0u;
  float sum[V] = {};
  uint32_t run = ~0u;      // the token whose rows are being summed
  bool from_front = false;  // ... since the chunk in front
  const auto finish = [&](bool leaves) {
    float* to = from_front ? s.front : leaves ? s.behind : nullptr;
    if (to) put_partial(to + (uint64_t)c * p.width + col, sum, n);
    else if (n != 0) put_row<TO>(p, run, col, n, sum);
  };
  for (uint32_t i0 = lo; i0 < hi; i0 += 64u) {
    const uint32_t i = min(i0 + lane, p.n_tokens - 1u);
    const uint32_t key = s.key[i], at = s.at[i];
    const uint32_t count = (uint32_t)__popcll(__ballot(i0 + lane < hi && key < p.vocab));  // those without gradient are last
    for (uint32_t j0 = 0; j0 < count; j0 += kBatch) {
      Vec<TI, V> x[kBatch];
#pragma unroll
      for (uint32_t j = 0; j < kBatch; ++j) {
        x[j] = {};
        if (j0 + j < count && n != 0) {
          const uint32_t t = __builtin_amdgcn_readlane(at, j0 + j);
          const TI* from = static_cast<const TI*>(p.grad_out) + (uint64_t)t * p.grad_out_ld + col;
          if (n == V) load<false>(x[j], from);
          else load_end(x[j], from, n, 0.f);
        }
      }
#pragma unroll
      for (uint32_t j = 0; j < kBatch; ++j) {
        if (j0 + j >= count) break;
        const uint32_t k = __builtin_amdgcn_readlane(key, j0 + j);
        if (k != run) {
          if (run != ~0u) finish(false);
          run = k, from_front = i0 + j0 + j == lo && k == before;
#pragma unroll
          for (int v = 0; v < V; ++v) sum[v] = 0.f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += x[j].get(v);
      }
    }
    if (count < 64u) break;
  }
  if (run != ~0u) finish(run == behind);
}

// Rows that go over chunk ends: the workgroup of the chunk where such a row starts adds its partial sums, eight wavefronts
// every eighth of them, then the eight sums in order.
constexpr uint32_t kJoinWaves = 8;
template <typename TO>
__global__ __launch_bounds__(64 * kJoinWaves) void k_token_joins(const EmbedGrad p, const Sums s) {
  __shared__ float part[kJoinWaves][64][4];
  const uint32_t c = blockIdx.x, lane = lane_id(), wave = threadIdx.x >> 6;
  const uint32_t lo = c * s.chunk, hi = lo + s.chunk;
  if (hi >= p.n_tokens) return;
  const uint32_t key = s.key[hi - 1u];
  if (key >= p.vocab || s.key[hi] != key) return;                       // no row leaves
  if (s.key[lo] == key && lo > 0 && s.key[lo - 1u] == key) return;        // it started further in front
  const uint32_t end = lower_bound(s.key, hi, p.n_tokens, key + 1u);      // the row's tokens are [.., end)
  const uint32_t last = (end - 1u) / s.chunk;                             // its last chunk
  const uint32_t col = (blockIdx.y * 64u + lane) * 4u;
  const uint32_t n = col < p.width ? min(4u, p.width - col) : 0u;
  float sum[4] = {};
  if (wave == 0) {
#pragma unroll
    for (uint32_t v = 0; v < 4; ++v)
      if (v < n) sum[v] = load1(s.behind + (uint64_t)c * p.width + col + v);
  }
#pragma unroll 4
  for (uint32_t d = c + 1u + wave; d <= last; d += kJoinWaves) {
#pragma unroll
    for (uint32_t v = 0; v < 4; ++v)
      if (v < n) sum[v] += load1(s.front + (uint64_t)d * p.width + col + v);
  }
#pragma unroll
  for (uint32_t v = 0; v < 4; ++v) part[wave][lane][v] = sum[v];
  __syncthreads();
  if (wave != 0 || n == 0) return;
#pragma unroll
  for (uint32_t w = 1; w < kJoinWaves; ++w)
#pragma unroll
    for (uint32_t v = 0; v < 4; ++v) sum[v] += part[w][lane][v];
  put_row<TO>(p, key, col, n, sum);
}

// A table without a token: zeros.
template <typename TO>
__global__ __launch_bounds__(kThreads) void k_token_none(const EmbedGrad p) {
  for (uint64_t row = blockIdx.x; row < p.vocab; row += gridDim.x)
    for (uint32_t col = threadIdx.x; col < p.width; col += kThreads)
      store1(static_cast<TO*>(p.grad) + row * p.grad_ld + col, from_f32<TO>(0.f));
}

// ---- launches ------------------------------------------------------------------------

uint32_t chunk_of(uint64_t n_tokens) {  // positions per chunk: 16, and about a thousand chunks where there are many
  uint64_t chunk = 16;
  while (chunk * 1024u < n_tokens) chunk *= 2;
  return (uint32_t)chunk;
}

struct Passes {
  uint32_t n, bits, blocks;
};
Passes passes_of(uint64_t n_tokens, uint64_t vocab) {
  uint32_t bits = 1;
  while (vocab >> bits) ++bits;  // keys 0 .. vocab
  const uint32_t n = (uint32_t)ceil_div(bits, kMaxDigitBits);
  return {n, (uint32_t)ceil_div(bits, n), (uint32_t)ceil_div(n_tokens, kSortBlock)};
}

struct Parts {  // offsets in bytes
  uint64_t key[2], at[2], counts, front, behind, total;
};
Parts parts_of(uint64_t n_tokens, uint64_t vocab, uint64_t width) {
  const Passes passes = passes_of(n_tokens, vocab);
  const uint64_t ids = round_up(4 * n_tokens, 256), rows = round_up(4 * width * ceil_div(n_tokens, chunk_of(n_tokens)), 256);
  Parts w{};
  for (int i = 0; i < 2; ++i) w.key[i] = 2 * i * ids, w.at[i] = (2 * i + 1) * ids;
  w.counts = 4 * ids;
  w.front = w.counts + round_up((uint64_t)passes.blocks * 4 << passes.bits, 256);
  w.behind = w.front + rows;
  w.total = w.behind + rows;
  return w;
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
  uint32_t* key[2] = {(uint32_t*)(base + w.key[0]), (uint32_t*)(base + w.key[1])};
  uint32_t* at[2] = {(uint32_t*)(base + w.at[0]), (uint32_t*)(base + w.at[1])};
  hipError_t e = with_id(token_dtype, [&](auto id) {
    typedef decltype(id) I;
    for (uint32_t i = 0; i < passes.n; ++i) {
      const Sort sort{key[(i + 1) & 1], at[(i + 1) & 1], key[i & 1], at[i & 1], (uint32_t*)(base + w.counts), i * passes.bits, passes.bits};
      if (i == 0) {
        hipLaunchKernelGGL((k_token_counts<I, true>), dim3(passes.blocks), dim3(kThreads), 0, s, p, sort);
        hipLaunchKernelGGL((k_token_move<I, true>), dim3(passes.blocks), dim3(kThreads), 0, s, p, sort, passes.blocks);
      } else {
        hipLaunchKernelGGL((k_token_counts<I, false>), dim3(passes.blocks), dim3(kThreads), 0, s, p, sort);
        hipLaunchKernelGGL((k_token_move<I, false>), dim3(passes.blocks), dim3(kThreads), 0, s, p, sort, passes.blocks);
      }
    }
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  const uint32_t last = (passes.n - 1) & 1;
  const uint32_t chunk = chunk_of(p.n_tokens), n_chunks = (uint32_t)ceil_div(p.n_tokens, chunk);
  const Sums sums{key[last], at[last], (float*)(base + w.front), (float*)(base + w.behind), chunk, n_chunks};
  return with_float(grad_dtype, [&](auto to) {
    typedef decltype(to) TO;
    e = with_float(grad_out_dtype, [&](auto ti) {
      typedef decltype(ti) TI;
      const uint32_t slabs = (uint32_t)ceil_div(p.width, 64u * (16u / sizeof(TI)));
      const uint32_t sum_blocks = (uint32_t)ceil_div((uint64_t)n_chunks * slabs, kWaves);
      const uint32_t clear_blocks = p.accumulate ? 0u : (uint32_t)ceil_div(p.vocab, 64u * kWaves);
      hipLaunchKernelGGL((k_token_sums<TI, TO>), dim3(sum_blocks + clear_blocks), dim3(kThreads), 0, s, p, sums, slabs, sum_blocks);
      return hipGetLastError();
    });
    if (e != hipSuccess || n_chunks < 2u) return e;
    hipLaunchKernelGGL((k_token_joins<TO>), dim3(n_chunks - 1u, (uint32_t)ceil_div(p.width, 256u)), dim3(64 * kJoinWaves), 0, s, p, sums);
    return hipGetLastError();
  });
}

}  // namespace lmt
