// Microscaled 4-bit values (OCP MXFP4): rounding, reading back, and grouped
// products on the block-scaled matrix instructions (layout and rules in
// lorex_block.h).
#include "lx_block.h"
#include "lx_vec.h"

#include <algorithm>
#include <type_traits>

namespace lx {
namespace {

constexpr int kBlk = 32;  // values under one scale

// ---------------------------------------------------------------- rounding
// Both directions are bound by memory (8 x 14336 rows of 4096 in bf16: rounding 252
// us, 4.7 TB/s, reading back 193 us, 6.2 TB/s), but for SwiGLU's exponential and
// quotient (32768 rows of 768 in bf16 42 us, 2.7 TB/s; 8192 of 14336 155, 3.4). A lane has 8 values of a row (4 lanes
// share a block of 32), TPR lanes a row, and U rows under way at once; there is no
// division by the row length.
template <int U, class F>
__device__ __forceinline__ void for_rows(int64_t rows, int vecs, int tpr, F&& f) {
  const int lt = threadIdx.x & (tpr - 1), rpb = 256 / tpr;
  for (int64_t r = (int64_t)blockIdx.x * rpb * U + (int)threadIdx.x / tpr; r < rows; r += (int64_t)gridDim.x * rpb * U)
    for (int v = lt; v < vecs; v += tpr) f(r, rpb, v * 8);
}

// Rounding: the largest magnitude of a block goes over its 4 lanes as bits: as
// unsigned integers magnitudes keep their order, and infinities and NaNs come
// out above every finite one. The conversion instruction divides by a power of
// two, rounds to nearest even and saturates at 6.
__device__ __forceinline__ uint32_t mx4_round(F8 x, int& s) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x.v[e]) & 0x7FFFFFFFu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true));
  const int e = (int)(top >> 23);  // biased; 255: infinity or NaN
  s = e == 255 ? 255 : e > 2 ? e - 2 : 0;
  // (2^-127 is not a normal number: there the values are doubled instead)
  const float f = __uint_as_float((uint32_t)(s > 0 ? s : 1) << 23);
#pragma unroll
  for (int j = 0; j < 8; ++j) x.v[j] = s > 0 ? x.v[j] : 2.f * x.v[j];
  uint32_t code = 0;
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x.v[0], x.v[1], f, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x.v[2], x.v[3], f, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x.v[4], x.v[5], f, 2);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x.v[6], x.v[7], f, 3);
  return s == 255 ? 0 : code;
}

template <int U, bool SWIGLU>
__global__ __launch_bounds__(256) void k_mx4_quantize(const Mx4Args a, int tpr) {
  const int Kp = LX_MX4_KP(a.K);
  for_rows<U>(a.rows, Kp / 8, tpr, [&](int64_t r, int rpb, int c) {
    Raw8 g[U], u[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t row = r + (int64_t)j * rpb;
      g[j] = u[j] = Raw8{};
      if (row < a.rows && c < a.K) {
        g[j] = load_raw8(a.x, a.f32, row * a.K * (SWIGLU ? 2 : 1) + c);
        if (SWIGLU) u[j] = load_raw8(a.x, a.f32, row * a.K * 2 + a.K + c);
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t row = r + (int64_t)j * rpb;
      F8 x = unpack8(g[j], a.f32);
      if (SWIGLU) {
        const F8 w = unpack8(u[j], a.f32);
#pragma unroll
        for (int e = 0; e < 8; ++e) x.v[e] = x.v[e] / (1.f + expf(-x.v[e])) * w.v[e];
      }
      int s;
      const uint32_t code = mx4_round(x, s);
      if (row < a.rows) {
        *(uint32_t*)(a.codes + row * (Kp / 2) + c / 2) = code;
        if ((c & (kBlk - 1)) == 0) a.scales[row * (Kp / kBlk) + c / kBlk] = (uint8_t)s;
      }
    }
  });
}

template <int U>
__global__ __launch_bounds__(256) void k_mx4_dequantize(const Mx4Args a, int tpr) {
  const int Kp = LX_MX4_KP(a.K);
  for_rows<U>(a.rows, a.K / 8, tpr, [&](int64_t r, int rpb, int c) {
    uint32_t code[U], s[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t row = r + (int64_t)j * rpb;
      code[j] = s[j] = 0;
      if (row < a.rows) {
        code[j] = *(const uint32_t*)(a.codes + row * (Kp / 2) + c / 2);
        s[j] = a.scales[row * (Kp / kBlk) + c / kBlk];
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t row = r + (int64_t)j * rpb;
      const float f = __uint_as_float(s[j] == 255 ? 0x7FC00000u : s[j] ? s[j] << 23 : 0x00400000u);
      F8 x;
      auto two = [&](auto sel, float& lo, float& hi) {
        const auto q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[j], 1.f, decltype(sel)::value);
        lo = q[0] * f;
        hi = q[1] * f;
      };
      two(std::integral_constant<int, 0>{}, x.v[0], x.v[1]);
      two(std::integral_constant<int, 1>{}, x.v[2], x.v[3]);
      two(std::integral_constant<int, 2>{}, x.v[4], x.v[5]);
      two(std::integral_constant<int, 3>{}, x.v[6], x.v[7]);
      if (row < a.rows) store8((void*)a.x, a.f32, row * a.K + c, x);
    }
  });
}

// ---------------------------------------------------------------- products
typedef int v8i __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v8i frag(const uint4& q) { return v8i{(int)q.x, (int)q.y, (int)q.z, (int)q.w, 0, 0, 0, 0}; }

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
__device__ __forceinline__ void group_rows(const Mx4GemmArgs& a, int g, int& lo, int& hi) {
  lo = hi = 0;
  if (g < a.G) {
    lo = min(max(a.offsets[g], 0), a.M);
    hi = min(max(a.offsets[g + 1], lo), a.M);
  }
}

// Row tiles over all groups (tiles of BM rows counted group by group).
template <int BM>
__device__ __forceinline__ int count_tiles(const Mx4GemmArgs& a) {
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
template <int BM>
__device__ __forceinline__ bool find_tile(const Mx4GemmArgs& a, int tile, int& g, int& m0, int& m1) {
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

// ---------------------------------------------------------------- few rows
// Four scale words of a row: 16 bytes at the words' own alignment. Read word by
// word they took half as long again as the codes (512 rows of 128 experts of 1536
// x 2048: 61 against 41 us).
typedef uint32_t vu4w __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t vu2h __attribute__((ext_vector_type(2), aligned(2)));

// 16 rows x 16 columns per wavefront for batches of few rows per group:
// bound by streaming the weights once. Both operands are read from memory in the
// layout of the 16x16x128 instruction (lane l holds row l % 16's block l / 16 of
// the 128 values of a step), 8 steps' loads in flight per wavefront; WK
// wavefronts of a workgroup share the K of the same columns where there are few
// columns, and add their sums in order. The weights are the instruction's first
// operand, so a lane ends with 4 consecutive columns of one output row.
template <int WK>
__global__ __launch_bounds__(256) void k_mx4_gemm_rows(const Mx4GemmArgs a) {
  constexpr int WN = 4 / WK;
  __shared__ float part[WK > 1 ? WK - 1 : 1][256];
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave % WK, wn = wave / WK;
  const int ntn = (a.N + 16 * WN - 1) / (16 * WN);
  const int rt = count_tiles<16>(a);
  const int cp = a.Kp / 2, sp = a.Kp / 32, steps = a.Kp / 128;
  Items it((int64_t)rt * ntn);
  for (; it.at < it.end; it.at += it.step) {
    // without groups the row tiles of the same columns follow each other
    const int64_t L = it.at;
    const int ti = (int)(a.offsets ? L / ntn : L % rt), n0 = (int)(a.offsets ? L % ntn : L / rt) * 16 * WN + wn * 16;
    int g, m0, m1;
    if (!find_tile<16>(a, ti, g, m0, m1)) return;
    const int m = m0 + l16;
    int arow = -1;
    if (m < m1) arow = a.row_map ? a.row_map[m] : m;
    if (arow >= a.a_rows) arow = -1;
    const int64_t brow = (int64_t)g * a.N + min(n0 + l16, a.N - 1);
    const uint8_t* const B = a.b + brow * cp + q * 16;
    const uint8_t* const Bs = a.bs + brow * sp;
    vf4 acc = {0.f, 0.f, 0.f, 0.f};
    // U steps from k on, all of this wavefront's: their loads, then their products
    auto batch = [&](auto count, int k) __attribute__((always_inline)) {
      constexpr int U = decltype(count)::value, UW = U < 4 ? 1 : U / 4;
      uint4 w[U], av[U];
      vu4 ws[UW], as[UW];
      auto words = [&](vu4(&v)[UW], const uint8_t* row) __attribute__((always_inline)) {
        if constexpr (U < 4) {
          v[0][0] = *(const uint32_t*)(row + k * 4);
        } else {
#pragma unroll
          for (int c = 0; c < UW; ++c) v[c] = *(const vu4w*)(row + k * 4 + c * 16);
        }
      };
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = *(const uint4*)(B + (int64_t)(k + u) * 64);
      words(ws, Bs);
#pragma unroll
      for (int u = 0; u < U; ++u) av[u] = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int c = 0; c < UW; ++c) as[c] = vu4{0, 0, 0, 0};
      if (arow >= 0) {
        const uint8_t* const A = a.a + (int64_t)arow * cp + q * 16;
#pragma unroll
        for (int u = 0; u < U; ++u) av[u] = *(const uint4*)(A + (int64_t)(k + u) * 64);
        words(as, a.as + (int64_t)arow * sp);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag(w[u]), frag(av[u]), acc, 4, 4, 0,
                                                               ws[u / 4][u & 3] >> (8 * q), 0, as[u / 4][u & 3] >> (8 * q));
    };
    const int k1 = (int)((int64_t)steps * (wk + 1) / WK);
    int k = (int)((int64_t)steps * wk / WK);
    for (; k + 8 <= k1; k += 8) batch(std::integral_constant<int, 8>{}, k);
    if (k + 4 <= k1) {
      batch(std::integral_constant<int, 4>{}, k);
      k += 4;
    }
    for (; k < k1; ++k) batch(std::integral_constant<int, 1>{}, k);
    if constexpr (WK > 1) {
      if (wk > 0) *(vf4*)&part[wk - 1][lane * 4] = acc;
      __syncthreads();
      if (wk == 0) {
#pragma unroll
        for (int v = 0; v < WK - 1; ++v) acc += *(const vf4*)&part[v][lane * 4];
      }
    }
    if (wk == 0 && m < m1) {
      if (arow < 0) acc = vf4{0.f, 0.f, 0.f, 0.f};  // (also where a weight is NaN)
      const int64_t at = (int64_t)m * a.N + n0 + q * 4;
      if (n0 + q * 4 + 4 <= a.N) {
        if (a.out_f32)
          *(vf4w*)((float*)a.out + at) = acc;
        else
          *(vu2h*)((uint16_t*)a.out + at) = vu2h{pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3])};
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (n0 + q * 4 + j < a.N) {
            if (a.out_f32)
              ((float*)a.out)[at + j] = acc[j];
            else
              ((uint16_t*)a.out)[at + j] = (uint16_t)pack_bf16(acc[j], 0.f);
          }
      }
    }
    if constexpr (WK > 1) __syncthreads();
  }
}

// ---------------------------------------------------------------- large tiles
typedef float f32x16 __attribute__((ext_vector_type(16)));
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

// BM x BN outputs per workgroup, a 2 x 2 grid of wavefronts (256 x 256: 2 x 4, two
// wavefronts per SIMD: one multiplies while the other waits for LDS or the barrier,
// and twice as many write results out; against 2 x 2 with twice the accumulators
// 8192 x 8192 x 2048 takes 87 for 97 us, 8192^3 283 for 288), 32x32x64
// instructions. Both operands go memory -> LDS directly in steps of 256 values
// (128 bytes a row, a whole cache line: 64 bytes a row took twice as long per
// byte), two steps in a ring, one streaming in while the other is multiplied.
// Inside a step's image the eight 16-byte chunks of a row are XORed with (row /
// 2) % 8, so the 16 lanes that a read serves together hit 16 different bank
// groups; a lane fetches the chunk that belongs at its LDS place. Scales come
// in groups of two steps (16 bytes a row) through a ring of two. The weights
// are the instruction's first operand: a lane ends with 4 consecutive columns
// of one row, which go through LDS into whole rows. 8192^3: 283 us, 3.9 PFLOP/s,
// the matrix units busy for 48% of the cycles at a clock that has fallen below 2 GHz
// (the instructions alone reach 6.5 from registers). Tried and slower: the two
// wavefronts of a SIMD half a phase apart (8192^3 297), scales read 16 bytes at a
// time without bank conflicts (301), the lines of the step after the next one
// touched ahead (5 to 20% more).
// SPLIT: an item is one of a.plan.splits parts of a tile's K (whole steps, an even
// number in all but the last), and its results are an fp32 [M][N] of its own, which
// a second launch adds up in order.
// Workgroups stay for several items: the next item's place and rows are looked
// up under the first loads of the present one, and its first loads are under way
// while the present one's results are written.
constexpr int tile_threads(int bm, int bn) { return bm * bn > 128 * 128 ? 512 : 256; }
constexpr int tile_groups_per_cu(int bm, int bn) { return bm * bn > 128 * 128 ? 1 : bm * bn == 128 * 128 ? 2 : 4; }

template <int BM, int BN, bool SPLIT>
__global__ __launch_bounds__(tile_threads(BM, BN), tile_groups_per_cu(BM, BN) * tile_threads(BM, BN) / 256)
void k_mx4_gemm_tile(const Mx4GemmArgs a) {
  constexpr int THR = tile_threads(BM, BN), NW = THR / 64, WC = NW / 2;
  constexpr int WM = BM / 2, WN = BN / WC, MI = WM / 32, NI = WN / 32;
  constexpr int RA = BM * 8 / THR, RB = BN * 8 / THR, R = RA + RB;  // 16-byte loads of a thread per step
  constexpr int STAGE = (BM + BN) * 128, SGRP = (BM + BN) * 16;
  constexpr int LDS = 2 * STAGE + 2 * SGRP + 16;  // (a half step reads a word past its scales)
  static_assert(LDS * tile_groups_per_cu(BM, BN) <= 160 * 1024, "");
  static_assert(NW * 32 * WN * 4 <= STAGE, "32 rows of each wavefront's results fit in a stage");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[LDS];

  const int ntn = (a.N + BN - 1) / BN;
  const int rt = count_tiles<BM>(a);
  Items it((int64_t)rt * ntn * (SPLIT ? a.plan.splits : 1));
  if (it.at >= it.end) return;

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int l32 = lane & 31, h = lane >> 5;
  const int wm = wave / WC, wn = wave % WC;
  const int cp = a.Kp / 2, sp = a.Kp / 32, full = a.Kp / 256;
  const bool odd = a.Kp & 128;  // a last step of 128 values

  struct Item {
    int m0, m1, n0;
    int split, t0, t1;               // steps t0 .. t1 - 1 of 256 values (t0 is even)
    bool tail;                       // and then the half step
    uint64_t there[(WM + 63) / 64];  // which of this wavefront's rows have a row of A
    const uint8_t *B, *Bs;           // the tile's first weight row and its scales
    uint32_t oa[RA];                 // a thread's byte offsets from A (the host sees to it that they fit
                                     // 32 bits)
    uint32_t qs;                     // its row of the scale groups: of A (threads below BM) or of B (the
                                     // last BN threads)
  };
  static_assert(BM + BN <= THR, "one row of scales per thread");
  // A's row for tile row r, -1 if there is none (past the tile, or a map entry out
  // of range): its loads read A's first row (the host sees to it that there is
  // one), its results are dropped or 0
  auto row_of = [&](const Item& q, int r) __attribute__((always_inline)) {
    const int m = q.m0 + r;
    if (m >= q.m1) return -1;
    const int src = a.row_map ? a.row_map[m] : m;
    return src >= 0 && src < a.a_rows ? src : -1;
  };
  // Item L: column tiles in bands of 8, so that what an XCD runs together shares
  // rows and weights in its L2.
  auto look_up = [&](int64_t L, Item& q) __attribute__((always_inline)) {
    q.split = 0;
    q.t0 = 0;
    q.t1 = full;
    q.tail = odd;
    if constexpr (SPLIT) {
      const int64_t all = (int64_t)rt * ntn;
      q.split = (int)(L / all);
      L -= q.split * all;
      q.t0 = q.split * a.plan.split_steps;
      q.t1 = min(q.t0 + a.plan.split_steps, full);
      q.tail = odd && q.split == a.plan.splits - 1;
    }
    const int64_t per_band = (int64_t)rt * 8;
    const int band = (int)(L / per_band), w = min(8, ntn - band * 8);
    const int rem = (int)(L - band * per_band), ti = rem / w;
    q.n0 = (band * 8 + rem - ti * w) * BN;
    int g = 0;
    q.m0 = q.m1 = 0;
    find_tile<BM>(a, ti, g, q.m0, q.m1);
    q.B = a.b + ((int64_t)g * a.N + q.n0) * cp;
    q.Bs = a.bs + ((int64_t)g * a.N + q.n0) * sp;
#pragma unroll
    for (int j = 0; j < RA; ++j) {
      const int r = (j * THR + tid) >> 3;
      q.oa[j] = (uint32_t)max(row_of(q, r), 0) * (uint32_t)cp + ((tid ^ (r >> 1)) & 7) * 16;
    }
    q.qs = (uint32_t)max(row_of(q, tid % BM), 0) * (uint32_t)sp;
#pragma unroll
    for (int j = 0; j < (WM + 63) / 64; ++j) q.there[j] = __ballot(row_of(q, wm * WM + j * 64 + lane) >= 0);
  };
  Item cur;
  // the offsets from B, formed when an item begins: they need no loads, and next
  // to the present item's they would not fit in registers
  uint32_t ob[RB];
  auto from_b = [&]() __attribute__((always_inline)) {
    const int last = a.N - 1 - cur.n0;
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const int r = (j * THR + tid) >> 3;
      ob[j] = (uint32_t)min(r, last) * (uint32_t)cp + ((tid ^ (r >> 1)) & 7) * 16;
    }
    if (wave >= NW - BN / 64) cur.qs = (uint32_t)min(tid % BN, last) * (uint32_t)sp;
  };
  // Group q of the scales: words 4 q .. 4 q + 3 of every row, 16 bytes a row (a
  // memory address need only be aligned to words). A row's last group holds its
  // last four words, so a step finds its words `late` words further on.
  const int words = sp / 4;
  auto late = [&](int q) __attribute__((always_inline)) { return words < 4 ? 0 : max(q * 4 - (words - 4), 0); };
  auto issue_scales = [&](int q) __attribute__((always_inline)) {
    uint8_t* const st = smem + 2 * STAGE + (q & 1) * SGRP;
    if (words >= 4) {
      const int at = (q * 4 - late(q)) * 4;
      if (wave < BM / 64) load_lds<16>(a.as + at, cur.qs, st + wave * 1024);
      if (wave >= NW - BN / 64) load_lds<16>(cur.Bs + at, cur.qs, st + BM * 16 + (wave - (NW - BN / 64)) * 1024);
    } else {
      // rows of fewer words: word by word, 16 rows x 4 words per load, the last
      // one repeated
      const int word = min(lane & 3, words - 1) * 4;
#pragma unroll 1
      for (int r0 = wave * 16; r0 < BM + BN; r0 += NW * 16) {
        const int r = r0 + (lane >> 2);
        if (r0 < BM)
          load_lds<4>(a.as, (uint32_t)max(row_of(cur, r), 0) * (uint32_t)sp + word, st + r0 * 16);
        else
          load_lds<4>(cur.Bs, (uint32_t)min(r - BM, a.N - 1 - cur.n0) * (uint32_t)sp + word, st + r0 * 16);
      }
    }
  };
  // load i of step t's operands into stage t % 2; in a half step the upper
  // chunks repeat the lower ones (they are not multiplied)
  auto issue_one = [&](int t, int i, bool half) __attribute__((always_inline)) {
    uint8_t* const st = smem + (t & 1) * STAGE;
    const int64_t at = (int64_t)t * 128;
    const int j = i < RA ? i : i - RA;
    const uint32_t back = half ? ((tid ^ (((j * THR + tid) >> 3) >> 1)) & 4) * 16 : 0;
    if (i < RA)
      load_lds<16>(a.a + at, cur.oa[j] - back, st + (j * NW + wave) * 1024);
    else
      load_lds<16>(cur.B + at, ob[j] - back, st + BM * 128 + (j * NW + wave) * 1024);
  };
  auto issue = [&](int t, bool half) __attribute__((always_inline)) {
    if ((t & 1) == 0) issue_scales(t >> 1);
#pragma unroll
    for (int i = 0; i < R; ++i) issue_one(t, i, half);
  };

  f32x16 acc[MI][NI];
  // a row's scales of a step are two words: a lane's block of instruction s is
  // 2 s + h, so after a shift by h bytes its scale is byte 0 or 2 of word s / 2
  const uint8_t* const la = smem + (wm * WM + l32) * 128;
  const uint8_t* const lb = smem + (BM + wn * WN + l32) * 128;
  const uint8_t* const lsa = smem + 2 * STAGE + (wm * WM + l32) * 16;
  const uint8_t* const lsb = smem + 2 * STAGE + (BM + wn * WN + l32) * 16;
  const int swz = (l32 >> 1) & 7;
  struct Scales {
    uint2 a[MI], b[NI];
  } sc, nx;
  uint4 fa[2][MI], fb[2][NI];
  auto read_scales = [&](Scales& q, int t) __attribute__((always_inline)) {
    const int st = ((t >> 1) & 1) * SGRP + (t & 1) * 8 + late(t >> 1) * 4;
    auto two = [&](const uint8_t* p) __attribute__((always_inline)) {
      return make_uint2(*(const uint32_t*)p, *(const uint32_t*)(p + 4));
    };
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) q.b[ni] = two(lsb + st + ni * 512);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) q.a[mi] = two(lsa + st + mi * 512);
  };
  auto shift_scales = [&](Scales& q) __attribute__((always_inline)) {
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) q.b[ni] = make_uint2(q.b[ni].x >> (8 * h), q.b[ni].y >> (8 * h));
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) q.a[mi] = make_uint2(q.a[mi].x >> (8 * h), q.a[mi].y >> (8 * h));
  };
  // fragments of instruction s of step t, into set s % 2
  auto read = [&](int s, int t) __attribute__((always_inline)) {
    const int c = (t & 1) * STAGE + ((2 * s + h) ^ swz) * 16;
    // (B's address from A's where a register less is what keeps the loop free of
    // scratch; elsewhere its own is 1% faster)
    const uint8_t *const pa = la + c, *const pb = THR == 512 ? pa + (BM + wn * WN - wm * WM) * 128 : lb + c;
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) fb[s & 1][ni] = *(const uint4*)(pb + ni * 4096);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) fa[s & 1][mi] = *(const uint4*)(pa + mi * 4096);
  };
  // The products of instruction s; from FIRST on, half of the loads of step t
  // between them: issued in one go they held up the products behind them. The
  // scheduling fences keep this order, and the reads of the next fragments
  // ahead of the products of the present ones.
  constexpr int kNone = R;
  auto multiply = [&](auto sv, auto first, int t) __attribute__((always_inline)) {
    constexpr int s = decltype(sv)::value, FIRST = decltype(first)::value;
    constexpr int P = MI * NI, H = R / 2;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int mi = i / NI, ni = i % NI;
      if constexpr (FIRST < R) {
        if (i * H / P < (i + 1) * H / P) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int l = i * H / P; l < (i + 1) * H / P; ++l) issue_one(t, FIRST + l, false);
      }
      acc[mi][ni] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
          frag(fb[s & 1][ni]), frag(fa[s & 1][mi]), acc[mi][ni], 4, 4, 2 * (s & 1), s < 2 ? sc.b[ni].x : sc.b[ni].y,
          2 * (s & 1), s < 2 ? sc.a[mi].x : sc.a[mi].y);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  using std::integral_constant;
  constexpr integral_constant<int, 0> i0{};
  constexpr integral_constant<int, 1> i1{};
  constexpr integral_constant<int, 2> i2{};
  constexpr integral_constant<int, 3> i3{};
  constexpr integral_constant<int, kNone> none{};

  // Step t > 0, entered when it has landed and step t - 1 has been read but for
  // its last products, which come first: under them and the next ones, step t + 1
  // is loaded into the place of step t - 1 (LOADS).
  auto step = [&](int t, auto loads) __attribute__((always_inline)) {
    constexpr bool LOADS = decltype(loads)::value;
    if (LOADS && (t & 1)) issue_scales((t + 1) >> 1);
    read_scales(nx, t);
    read(0, t);
    multiply(i3, integral_constant<int, LOADS ? 0 : kNone>{}, t + 1);
    sc = nx;
    shift_scales(sc);
    read(1, t);
    multiply(i0, integral_constant<int, LOADS ? R / 2 : kNone>{}, t + 1);
    read(2, t);
    multiply(i1, none, 0);
    read(3, t);
    multiply(i2, none, 0);
    land_and_meet();
  };
  look_up(it.at, cur);
  from_b();
  issue(cur.t0, cur.t0 == full);
  for (;;) {
    it.at += it.step;
    const bool more = it.at < it.end;
    Item next;
    if (more) look_up(it.at, next);
    land_and_meet();
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x16{};
    int t = cur.t0;
    const int t1 = cur.t1;
    if (t < t1) {
      if (t + 1 < t1 || cur.tail) issue(t + 1, t + 1 == full);
      read_scales(sc, t);
      read(0, t);
      shift_scales(sc);
      read(1, t);
      multiply(i0, none, 0);
      read(2, t);
      multiply(i1, none, 0);
      read(3, t);
      multiply(i2, none, 0);
      land_and_meet();
      for (++t; t + 1 < t1; ++t) step(t, std::true_type{});
      if (t < t1) {
        if (cur.tail) issue(full, true);
        step(t, std::false_type{});
      }
      multiply(i3, none, 0);
    }
    if (cur.tail) {
      read_scales(sc, full);
      read(0, full);
      shift_scales(sc);
      read(1, full);
      multiply(i0, none, 0);
      multiply(i1, none, 0);
      land_and_meet();  // (the ring is free)
    }

    const int m0 = cur.m0, m1 = cur.m1, nb = cur.n0 + wn * WN;
    uint64_t there[(WM + 63) / 64];
#pragma unroll
    for (int j = 0; j < (WM + 63) / 64; ++j) there[j] = cur.there[j];
    void* const out = SPLIT ? (void*)(a.part + (int64_t)cur.split * a.M * a.N) : a.out;
    const bool out_f32 = SPLIT || a.out_f32;
    if (more) {
      cur = next;
      from_b();
      issue(cur.t0, cur.t0 == full);
    }

    // 32 rows at a time through this wavefront's part of stage 1 (the next item's
    // first step is on its way into stage 0), 16-byte chunks XORed by the row, and
    // out as whole rows of WN columns (the empty asm keeps the addresses from being
    // formed before the loop, where they would not fit in registers)
    int ln = lane;
    asm volatile("" : "+v"(ln));
    constexpr int LPR = WN / 8;  // lanes of a row
    uint8_t* const e = smem + STAGE + wave * 32 * WN * 4;
    auto chunk = [](int r, int c) { return r * WN * 4 + (c ^ (WN == 32 ? (r >> 1) & 7 : r & 15)) * 16; };
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(vf4*)(e + chunk(ln & 31, ni * 8 + 2 * q + (ln >> 5))) =
              vf4{acc[mi][ni][4 * q], acc[mi][ni][4 * q + 1], acc[mi][ni][4 * q + 2], acc[mi][ni][4 * q + 3]};
      asm volatile("" ::: "memory");  // (a wavefront's LDS accesses run in order)
#pragma unroll 4
      for (int r0 = 0; r0 < 32; r0 += 64 / LPR) {
        const int r = r0 + ln / LPR, wr = mi * 32 + r, m = m0 + wm * WM + wr, c = nb + ln % LPR * 8;
        const vf4 u = *(const vf4*)(e + chunk(r, ln % LPR * 2)), v = *(const vf4*)(e + chunk(r, ln % LPR * 2 + 1));
        if (m < m1 && c < a.N) {
          F8 o{{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]}};
          if (!(there[mi / 2] >> (wr & 63) & 1)) o = F8{};
          const int64_t at = (int64_t)m * a.N + c;
          if (c + 8 <= a.N) {
            store8_any(out, out_f32, at, o);
          } else {
#pragma unroll
            for (int k = 0; k < 7; ++k)
              if (c + k < a.N) {
                if (out_f32)
                  ((float*)out)[at + k] = o.v[k];
                else
                  ((uint16_t*)out)[at + k] = (uint16_t)pack_bf16(o.v[k], 0.f);
              }
          }
        }
      }
      asm volatile("" ::: "memory");
    }
    if (!more) break;
  }
}

// The parts' sums, in order, for the rows that belong to a group.
__global__ __launch_bounds__(256) void k_mx4_gemm_sum(const Mx4GemmArgs a) {
  const int lo = a.offsets ? min(max(a.offsets[0], 0), a.M) : 0, hi = a.offsets ? min(max(a.offsets[a.G], lo), a.M) : a.M;
  const int64_t first = (int64_t)lo * a.N, end = (int64_t)hi * a.N, all = (int64_t)a.M * a.N;
  for (int64_t i = first + ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < end; i += (int64_t)gridDim.x * 1024) {
    const int n = (int)min(end - i, (int64_t)4);
    vf4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.plan.splits; ++s) {
      const float* const p = a.part + s * all + i;
      if (n == 4)
        v += *(const vf4w*)p;
      else
        for (int j = 0; j < n; ++j) v[j] += p[j];
    }
    if (a.out_f32) {
      if (n == 4)
        *(vf4w*)((float*)a.out + i) = v;
      else
        for (int j = 0; j < n; ++j) ((float*)a.out)[i + j] = v[j];
    } else if (n == 4) {
      *(vu2h*)((uint16_t*)a.out + i) = vu2h{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
      for (int j = 0; j < n; ++j) ((uint16_t*)a.out)[i + j] = (uint16_t)pack_bf16(v[j], 0.f);
    }
  }
}

}  // namespace

// Lanes of a row for `vecs` groups of 8 values, workgroups for U rows at a time.
static int row_lanes(int vecs) {
  int n = 1;
  while (n < vecs && n < 256) n *= 2;
  return n;
}
static int row_grid(int64_t rows, int tpr, int U) {
  const int64_t per = 256 / tpr * U;
  return (int)std::min<int64_t>((rows + per - 1) / per, 1 << 16);
}

hipError_t launch_mx4_quantize(const Mx4Args& a, hipStream_t s) {
  const int tpr = row_lanes(LX_MX4_KP(a.K) / 8);
  // four rows under way where that still leaves several workgroups per compute
  // unit
  const bool many = row_grid(a.rows, tpr, 4) >= 2048;
  const int grid = row_grid(a.rows, tpr, many ? 4 : 1);
  if (a.swiglu)
    many ? k_mx4_quantize<4, true><<<grid, 256, 0, s>>>(a, tpr) : k_mx4_quantize<1, true><<<grid, 256, 0, s>>>(a, tpr);
  else
    many ? k_mx4_quantize<4, false><<<grid, 256, 0, s>>>(a, tpr) : k_mx4_quantize<1, false><<<grid, 256, 0, s>>>(a, tpr);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const Mx4Args& a, hipStream_t s) {
  const int tpr = row_lanes(a.K / 8);
  const bool many = row_grid(a.rows, tpr, 4) >= 2048;
  const int grid = row_grid(a.rows, tpr, many ? 4 : 1);
  many ? k_mx4_dequantize<4><<<grid, 256, 0, s>>>(a, tpr) : k_mx4_dequantize<1><<<grid, 256, 0, s>>>(a, tpr);
  return hipGetLastError();
}

template <int BM, int BN, bool SPLIT = false>
static hipError_t launch_tile(const Mx4GemmArgs& a, hipStream_t s) {
  const int64_t tiles = a.offsets ? std::min<int64_t>((int64_t)a.M / BM + a.G, a.M) : ((int64_t)a.M + BM - 1) / BM;
  const int64_t items = tiles * (((int64_t)a.N + BN - 1) / BN) * (SPLIT ? a.plan.splits : 1);
  const int64_t most = 256 * tile_groups_per_cu(BM, BN);
  k_mx4_gemm_tile<BM, BN, SPLIT><<<(unsigned)std::min((items + 7) / 8 * 8, most), tile_threads(BM, BN), 0, s>>>(a);
  return hipGetLastError();
}

template <int WK>
static hipError_t launch_rows(const Mx4GemmArgs& a, hipStream_t s) {
  constexpr int BM = 16, BN = 16 * (4 / WK);
  const int64_t tiles = a.offsets ? std::min<int64_t>((int64_t)a.M / BM + a.G, a.M) : ((int64_t)a.M + BM - 1) / BM;
  const int64_t items = tiles * (((int64_t)a.N + BN - 1) / BN);
  k_mx4_gemm_rows<WK><<<(unsigned)std::min<int64_t>((items + 7) / 8 * 8, 1 << 16), 256, 0, s>>>(a);
  return hipGetLastError();
}

// Which kernel. Rows of a group are not known here, only their mean.
//   at most 16 rows: the row kernel, K shared by four wavefronts where K is long
//     and columns are few (4096 columns, K = 14336: 10.1 against 20.3 us alone;
//     2048 x 2048: 8.4 against 7.1)
//   else the tile that leaves the fullest compute unit the least work: a 256 x 256
//     tile counts 0.88, one of 128 x 128 0.3 and one of 64 x 64 0.1, what they take
//     next to each other on a full machine (4096^3, 1024 tiles of 128 x 128: 55
//     against 46 us; 8192 rows of 16 experts of 4096 x 4096 126 against 117; 6144 x
//     6144 x 4096 119 against 113; 128 experts of 1536 x 2048, 32768 rows, 64 x 64 186
//     against 128 x 128 144); a group's last tile is taken to be half full, which
//     errs where groups have a little less than a tile (24576 rows of the 128
//     experts, 192 each: 256 x 256 111, 128 x 128 100). So 512 x 14336 x 4096 runs
//     on 448 tiles of 128 x 128 (26 us) and not on 112 of 256 x 256 (35), and 512 rows
//     of the 128 experts on 64 x 64 ones (40, 128 x 128 45, row kernel 44 to 47)
//   64 x 64 tiles that would leave half the machine idle over a long K share it (64
//     x 4096 x 14336, 64 tiles: 35 us, in four parts 16; not yet at K = 4096, where
//     the second launch takes more than the parts save: 9 against 12)
Mx4GemmPlan mx4_gemm_plan(int M, int N, int Kp, int G) {
  Mx4GemmPlan p{};
  p.splits = 1;
  if (M <= 16) {
    const int64_t waves = ((int64_t)N + 15) / 16 * std::min(M, G);
    p.kernel = waves <= 1024 && Kp >= 4096 ? Mx4GemmPlan::kRows4 : Mx4GemmPlan::kRows;
    return p;
  }
  const int64_t groups = std::min(M, G);
  auto tiles = [&](int64_t b) { return (G > 1 ? (M + groups * (b / 2)) / b : (M + b - 1) / b) * (((int64_t)N + b - 1) / b); };
  auto load = [&](int64_t b, double weight) { return (double)((tiles(b) + 255) / 256) * weight; };
  const double w256 = load(256, 0.88), w128 = load(128, 0.3), w64 = load(64, 0.1);
  if (w256 < w128 && w256 < w64) {
    p.kernel = Mx4GemmPlan::kTile256;
  } else if (w128 <= w64) {
    p.kernel = Mx4GemmPlan::kTile128;
  } else {
    p.kernel = Mx4GemmPlan::kTile64;
    const int full = Kp / 256;
    const int64_t s = std::min<int64_t>(256 / std::max<int64_t>(tiles(64), 1), full / 8);
    if (s > 1 && full >= 24) {
      p.split_steps = (int)((full + s - 1) / s + 1) & ~1;
      p.splits = (full + p.split_steps - 1) / p.split_steps;
    }
  }
  return p;
}

hipError_t launch_mx4_gemm(const Mx4GemmArgs& a, hipStream_t s) {
  switch (a.plan.kernel) {
    case Mx4GemmPlan::kRows4: return launch_rows<4>(a, s);
    case Mx4GemmPlan::kRows: return launch_rows<1>(a, s);
    case Mx4GemmPlan::kTile256: return launch_tile<256, 256>(a, s);
    case Mx4GemmPlan::kTile128: return launch_tile<128, 128>(a, s);
    default: return a.plan.splits > 1 ? launch_tile<64, 64, true>(a, s) : launch_tile<64, 64>(a, s);
  }
}

hipError_t launch_mx4_gemm_sum(const Mx4GemmArgs& a, hipStream_t s) {
  const int64_t n = ((int64_t)a.M * a.N + 1023) / 1024;
  k_mx4_gemm_sum<<<(unsigned)std::min<int64_t>(n, 1 << 16), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lx
