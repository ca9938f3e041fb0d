// What the products per group of rows share: the row tiles of the groups, the order
// in which workgroups take them, and loads from memory to LDS.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lx {

// Inclusive prefix sum over the 64 lanes (all active): row shifts within 16
// lanes, then the totals of the rows before.
__device__ __forceinline__ int lane_prefix(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  const int r0 = __builtin_amdgcn_readlane(x, 15), r1 = __builtin_amdgcn_readlane(x, 31),
            r2 = __builtin_amdgcn_readlane(x, 47), row = (threadIdx.x & 63) >> 4;
  return x + (row >= 1 ? r0 : 0) + (row >= 2 ? r1 : 0) + (row >= 3 ? r2 : 0);
}

// A group's rows, clamped to [0, M].
template <class A>
__device__ __forceinline__ void group_rows(const A& a, int g, int& lo, int& hi) {
  lo = hi = 0;
  if (g < a.G) {
    lo = min(max(a.offsets[g], 0), a.M);
    hi = min(max(a.offsets[g + 1], lo), a.M);
  }
}

// Row tiles over all groups (tiles of BM rows counted group by group).
template <int BM, class A>
__device__ __forceinline__ int count_tiles(const A& a) {
  if (!a.offsets) return (a.M + BM - 1) / BM;
  int n = 0;
#pragma unroll 4
  for (int g0 = 0; g0 < a.G; g0 += 64) {
    int lo, hi;
    group_rows(a, g0 + (threadIdx.x & 63), lo, hi);
    n += (hi - lo + BM - 1) / BM;
  }
  return __builtin_amdgcn_readlane(lane_prefix(n), 63);
}

// The group and the rows of row tile `tile`, found by each wavefront: 64 groups
// at a time, a prefix sum of their tile counts over the lanes. false: there is no
// such tile. All results are uniform.
template <int BM, class A>
__device__ __forceinline__ bool find_tile(const A& a, int tile, int& g, int& m0, int& m1) {
  if (!a.offsets) {
    g = 0;
    m0 = tile * BM;
    m1 = min(m0 + BM, a.M);
    return m0 < a.M;
  }
#pragma unroll 4
  for (int g0 = 0; g0 < a.G; g0 += 64) {
    int lo, hi;
    group_rows(a, g0 + (threadIdx.x & 63), lo, hi);
    const int n = (hi - lo + BM - 1) / BM, sum = lane_prefix(n), all = __builtin_amdgcn_readlane(sum, 63);
    if (tile < all) {
      const int src = __builtin_ctzll(__ballot(tile < sum));
      g = g0 + src;
      m0 = __builtin_amdgcn_readlane(lo, src) + (tile - __builtin_amdgcn_readlane(sum - n, src)) * BM;
      m1 = min(m0 + BM, __builtin_amdgcn_readlane(hi, src));
      return true;
    }
    tile -= all;
  }
  return false;
}

// The work items of one workgroup: workgroups go round the 8 XCDs, and XCD x
// takes a contiguous range of all items.
struct Items {
  int64_t at, end, step;
  __device__ __forceinline__ Items(int64_t all) {
    const int x = blockIdx.x & 7;
    const int64_t per = all / 8, rest = all % 8, first = x * per + min((int64_t)x, rest);
    at = first + (blockIdx.x >> 3);
    end = first + per + (x < rest);
    step = gridDim.x >> 3;
  }
};

typedef __attribute__((address_space(3))) void lds_void_t;

// One direct memory -> LDS load per lane: lane i fills LDS bytes [dst + SIZE i,
// + SIZE) from base + its own 32-bit byte offset (base and dst are uniform).
// Inline asm, so that the only waits on it are the ones written below; M0 is
// written here only, and the s_nop is the wait state that the load needs after
// a write of M0.
template <int SIZE>
__device__ __forceinline__ void load_lds(const void* base, uint32_t off, const void* dst) {
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)dst);
  if constexpr (SIZE == 16)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory");
}

// All of this wavefront's loads have landed and its LDS reads are done, then
// every wavefront's.
__device__ __forceinline__ void land_and_meet() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

}  // namespace lx
