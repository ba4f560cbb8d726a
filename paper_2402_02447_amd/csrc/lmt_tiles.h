// What the tiled products of lmt.h share: the shape of a tile, which tile a workgroup has, and how operands get to LDS.
#ifndef LMT_TILES_H_
#define LMT_TILES_H_

#include "lmt_device.h"

namespace lmt {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// Of a list of n items: the one for workgroup `id`.  XCD x, which takes every eighth workgroup, gets an eighth of the list, so that its
// L2 sees neighbours.
__device__ __forceinline__ uint64_t neighbours(uint64_t id, uint64_t n) {
  constexpr uint32_t kXcds = 8;
  const uint64_t x = id % kXcds, share = n / kXcds, extra = n % kXcds;
  return x * share + min(x, extra) + id / kXcds;
}

// A tile of c for WM x WN wavefronts, each with TM x TN squares of 32 x 32.  k goes through LDS in blocks of 128 bytes a row, two at
// a time: one that is being multiplied and one on its way.  With eight wavefronts, two on a SIMD, they go in two groups that
// take turns: one multiplies 64 bytes of k while the other reads its next operands from LDS.
template <int WM_, int WN_, int TM_, int TN_>
struct Shape {
  static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_;
  static constexpr int waves = WM * WN, threads = 64 * waves;
  static constexpr int rows_m = 32 * TM * WM, rows_n = 32 * TN * WN;  // of c
  static constexpr int rows = rows_m + rows_n;                        // staged: a's, then b's
  static constexpr int loads = rows * 8 / threads;                    // of 16 bytes per thread and block
  static constexpr int lds = 2 * rows * 128;                          // stages; then results, 64 x 64 per wavefront
  static constexpr bool turns = waves == 8;
  static_assert(rows_m % (8 * waves) == 0 && rows_n % (8 * waves) == 0, "a load of all wavefronts is a's or b's");
  static_assert(TN == 2 && TM % 2 == 0 && lds >= waves * 64 * 64 * 4, "results go out by squares of 64 x 64");
};

// Which tile a workgroup has: a list of tiles that goes down kGroup tiles of m, then across n, so that both operands of the tiles in
// flight on an XCD are few.
struct Tiles {
  uint32_t across, down, splits, split_blocks;  // of c in n and m; parts of k, and blocks of 128 in each
};
constexpr uint32_t kGroup = 8;
__device__ __forceinline__ void tile_of(const Tiles& t, uint32_t id, uint32_t* tm, uint32_t* tn) {
  id = (uint32_t)neighbours(id, t.across * t.down);
  const uint32_t group = id / (kGroup * t.across), tall = min(kGroup, t.down - group * kGroup), in_group = id - group * kGroup * t.across;
  *tm = group * kGroup + in_group % tall, *tn = in_group / tall;
}

// What has been added is added here: the compiler would put the instructions off, their operands in registers until then.
template <typename S>
__device__ __forceinline__ void settle(f32x16 (&acc)[S::TM][S::TN]) {
#pragma unroll
  for (int i = 0; i < S::TM; ++i)
#pragma unroll
    for (int j = 0; j < S::TN; ++j) asm volatile("" : "+v"(acc[i][j]));
  __builtin_amdgcn_sched_barrier(0);
}
// Buffer loads from `base` on: a 32-bit offset per lane and one per wavefront, without address arithmetic.
__device__ __forceinline__ uint32_t load_word(const uint8_t* base, uint32_t offset, uint32_t wave_offset) {
  return __builtin_amdgcn_raw_buffer_load_b32(__builtin_amdgcn_make_buffer_rsrc((void*)base, 0, -1, 0x27000), (int)offset, (int)wave_offset, 0);
}
// ... of 16 bytes per lane, which go to lds + 16 * lane.
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t offset, uint32_t wave_offset, uint8_t* lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void*)base, 0, -1, 0x27000), (__attribute__((address_space(3))) void*)lds, 16, (int)offset, (int)wave_offset, 0, 0);
}
// A number that is the same in all lanes, in a scalar register: what is made by a division, for one, is not there by itself.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
// The same, without the compiler's knowledge: it waits for every load to LDS in front of every read of LDS that could be of the same
// place, and does not see that buffers take turns.  So whoever reads what was sent waits for it himself (wait_and_meet).  No register is written, and the
// operands are read when the instruction is issued.  Scalar registers that a vector instruction wrote (a lane read into one) may be read by a load five
// wait states later, which the compiler sees to for its own instructions alone: hence s_nop 4, which covers m0's one as well.
__device__ __forceinline__ void send_to_lds(const uint8_t* base, uint32_t offset, uint32_t wave_offset, uint8_t* lds) {
  const uint64_t at = (uint64_t)(uintptr_t)base;
  const u32x4 rsrc = {uniform((uint32_t)at), uniform((uint32_t)(at >> 32)) & 0xffffu, 0xffffffffu, 0x27000u};
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"{m0}"((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds), "v"(offset), "s"(rsrc),
               "s"(uniform(wave_offset))
               : "memory");
}
// At most N of this wavefront's loads are in flight and none of its LDS reads; then a barrier.  (A barrier alone does not order memory
// operations for the compiler, a fence would wait for all loads.)
template <int N>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

__device__ __forceinline__ void reads_done_and_meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void meet() { asm volatile("s_barrier" ::: "memory"); }

}  // namespace
}  // namespace lmt
#endif  // LMT_TILES_H_
