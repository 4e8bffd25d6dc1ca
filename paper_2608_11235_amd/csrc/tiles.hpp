// What the tiled products share: loads straight into LDS, their waits, and the order of the tiles.
#pragma once
#include "common.hpp"

namespace cora {

constexpr int GROUP_M = 8;  // M tiles walked before the next N tile (see tile_of)

template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// 16 bytes per lane from buffer offset voff + soff straight into LDS: lane l's bytes land at
// lds_off + 16 l.  Inline asm, because the compiler would wait for every such load before
// the next LDS read; it has no register output.
__device__ __forceinline__ void load_lds(uint32_t lds_off, int voff, u32x4_t rs, int soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds_off),
               "v"(voff), "s"(rs), "s"(soff)
               : "memory", "m0");
}

// the same of 4 bytes per lane
__device__ __forceinline__ void load_lds_dword(uint32_t lds_off, int voff, u32x4_t rs, int soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(lds_off),
               "v"(voff), "s"(rs), "s"(soff)
               : "memory", "m0");
}

__device__ __forceinline__ u32x4_t buffer_rsrc(const void* p, int64_t bytes) {
  const uint64_t a = (uint64_t)p;
  return u32x4_t{(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu,
                 (uint32_t)(bytes > 0xffffffffLL ? 0xffffffffLL : bytes), 0x00020000u};
}

// Tile of logical index t: N tiles in order, all M tiles (at most GROUP_M at a time) of one
// before the next.  xcd_remap hands each XCD a contiguous run of that order, so the tiles an
// XCD runs at once cover about as many M as N tiles and share both operands in its L2
// (at 16 M tiles, 4096 x 37888 x 3584: 970 -> 949 us).
__device__ __forceinline__ void tile_of(int t, int num_m, int n_tiles, int& tm, int& tn) {
  if (num_m <= GROUP_M) {
    tm = t % num_m;
    tn = t / num_m;
    return;
  }
  const int per = GROUP_M * (n_tiles / num_m), grp = t / per, first = grp * GROUP_M;
  const int gm = min(GROUP_M, num_m - first), r = t - grp * per;
  tm = first + r % gm;
  tn = r / gm;
}

}  // namespace cora
