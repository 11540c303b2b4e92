// What the tile kernels of products share: loads from memory straight into LDS, waits for them, the order of the tiles.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tsenor_dev {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

// keeps the instructions around it in the order written
#define TSENOR_IN_ORDER() __builtin_amdgcn_sched_barrier(0)

struct Resource {
  uint64_t base;
  uint32_t bytes, format;
};
__device__ __forceinline__ intx4 resource_of(const void* base, int64_t bytes) {
  return __builtin_bit_cast(intx4, Resource{(uint64_t)base, (uint32_t)bytes, 0x00020000u});
}
// 16 (or 4) bytes per lane from memory into LDS, in the order of the lanes from byte `to` on.  (The compiler would wait for loads into
// LDS that it knows of before any read of LDS; here the waits stand in the code.  A scalar write of m0 needs one other
// instruction before such a load.)
__device__ __forceinline__ void load_to_lds(uint32_t to, int lane_offset, const intx4& from, int offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(lane_offset), "s"(from), "s"(offset)
               : "memory", "m0");
}
__device__ __forceinline__ void load_dword_to_lds(uint32_t to, int lane_offset, const intx4& from, int offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(to), "v"(lane_offset), "s"(from), "s"(offset)
               : "memory", "m0");
}
// waits for what this wave has asked of LDS (with LDS), and of memory but for the last PENDING loads, then for the other waves
template <int PENDING, bool LDS = true>
__device__ __forceinline__ void meet() {
  static_assert(PENDING < 64);
  __builtin_amdgcn_s_waitcnt((LDS ? 0x0070 : 0x0F70) | (PENDING & 15) | (PENDING >> 4) << 14);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");  // (neither of the two keeps a read of LDS behind it)
  TSENOR_IN_ORDER();
}
constexpr int kAnyPending = 63;

// Which tile a workgroup takes: the ones that run on an XCD at a time (workgroups go round the eight) are neighbours, four rows of
// tiles high, and share its L2.  (14336 x 4096 x 8192: 374 us; 2 high 390, 8 high 376, 16 high 379, without XCDs 385-400.)
constexpr int kXcds = 8, kTilesHigh = 4;
__device__ __forceinline__ void tile_of(int id, int tiles_m, int tiles_n, int& tile_m, int& tile_n) {
  const int total = tiles_m * tiles_n, per = total / kXcds, rest = total % kXcds, xcd = id % kXcds;
  id = xcd * per + min(xcd, rest) + id / kXcds;
  const int first = id / (kTilesHigh * tiles_n) * kTilesHigh, high = min(kTilesHigh, tiles_m - first), at = id - first * tiles_n;
  tile_m = first + at % high, tile_n = at / high;
}

}  // namespace tsenor_dev
