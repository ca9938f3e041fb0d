// Products of 8-bit activations and 4-bit weights per group of rows, with bias,
// activation and residual (formulas and layout in lorex_block.h), on the
// block-scaled matrix instructions with one operand e2m1 and the other e4m3.
#include "lx_block.h"
#include "lx_groups.h"
#include "lx_mx8.h"
#include "lx_silu.h"
#include "lx_vec.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace lx {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef uint32_t vu4w __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t vu2h __attribute__((ext_vector_type(2), aligned(2)));

__device__ __forceinline__ v8i frag4(const vu4& q) { return v8i{(int)q[0], (int)q[1], (int)q[2], (int)q[3], 0, 0, 0, 0}; }
__device__ __forceinline__ v8i frag8(const vu4& p, const vu4& q) {
  return v8i{(int)p[0], (int)p[1], (int)p[2], (int)p[3], (int)q[0], (int)q[1], (int)q[2], (int)q[3]};
}

// The instruction adds up 16 products at a time and drops what lies more than 13 bits
// below the largest product's exponents: e4m3 reaches over 18 binades, and a few of
// its bits are lost then (the sums of normal values are off by 1e-5 of their size, and
// what is left of large products that cancel by all of it; with both operands e2m1
// nothing is). Activations whose exponent field's top bit is
// set (from 2 on under the block's scale) and the others are within the window among
// themselves, so two instructions, one for each, drop nothing.
template <bool HI>
__device__ __forceinline__ v8i half_of(v8i a) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t m = ((uint32_t)a[j] >> 6) & 0x01010101u, mask = (m << 8) - m;
    a[j] &= (int)(HI ? mask : ~mask);
  }
  return a;
}

// ---------------------------------------------------------------- epilogue
__device__ __forceinline__ float value(const void* p, bool f32, int64_t i) {
  return f32 ? ((const float*)p)[i] : __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
}
// n (1 .. 4) consecutive values at a place that is only aligned to its type.
__device__ __forceinline__ vf4 load4_any(const void* p, bool f32, int64_t i, int n) {
  vf4 r = {0.f, 0.f, 0.f, 0.f};
  if (n >= 4) {
    if (f32) return *(const vf4w*)((const float*)p + i);
    const vu2h b = *(const vu2h*)((const uint16_t*)p + i);
    return vf4{__uint_as_float(b[0] << 16), __uint_as_float(b[0] & 0xFFFF0000u), __uint_as_float(b[1] << 16),
               __uint_as_float(b[1] & 0xFFFF0000u)};
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (j < n) r[j] = value(p, f32, i + j);
  return r;
}

// The activation's arguments, 4 columns from c on: product and bias. `there`: the row
// exists in A (else the product is 0, whatever the weights hold).
__device__ __forceinline__ vf4 with_bias(const Mx8GemmArgs& a, int g, int c, int n, bool there, vf4 z) {
  if (!there) z = vf4{0.f, 0.f, 0.f, 0.f};
  if (a.bias && n > 0) z += load4_any(a.bias, a.bias_f32, (int64_t)g * a.N + c, n);
  return z;
}
__device__ __forceinline__ vf4 activate(int act, vf4 z) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (act == LX_ACT_SILU) z[j] = silu(z[j]);
    if (act == LX_ACT_GELU) z[j] = 0.5f * z[j] * erfcf(z[j] * -0.70710678118654752f);
  }
  return z;
}
__device__ __forceinline__ vf4 swiglu(vf4 z, vf4 u) {
#pragma unroll
  for (int j = 0; j < 4; ++j) z[j] = silu(z[j]) * u[j];
  return z;
}

// 8 columns from c on of row m: residual, rounding, store. Four consecutive lanes
// (all active) hold a block of 32 columns that begins at a multiple of 32.
template <bool MX8>
__device__ __forceinline__ void finish(const Mx8GemmArgs& a, int64_t m, int c, bool row, F8 x) {
  const bool whole = c + 8 <= a.cols;
  if (a.res && row) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int n = min(a.cols - c - 4 * h, 4);
      if (n > 0) {
        const vf4 r = load4_any(a.res, a.res_f32, m * a.cols + c + 4 * h, n);
#pragma unroll
        for (int j = 0; j < 4; ++j) x.v[4 * h + j] += r[j];
      }
    }
  }
  if constexpr (MX8) {
    if (c >= a.cols) x = F8{};  // the row's padding (cols is a multiple of 8)
    int s;
    const uint2 code = mx8_round(x, s);
    const int colsp = LX_MX8_KP(a.cols);
    if (row && c < colsp) {
      *(uint2*)((uint8_t*)a.out + m * colsp + c) = code;
      if ((c & 31) == 0) a.out_scales[m * (colsp / 32) + c / 32] = (uint8_t)s;
    }
  } else if (row && whole) {
    store8_any(a.out, a.out_f32, m * a.cols + c, x);
  } else if (row) {
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (c + j < a.cols) {
        if (a.out_f32)
          ((float*)a.out)[m * a.cols + c + j] = x.v[j];
        else
          ((uint16_t*)a.out)[m * a.cols + c + j] = (uint16_t)pack_bf16(x.v[j], 0.f);
      }
  }
}

// ---------------------------------------------------------------- few rows
// 16 rows x 16 columns per wavefront for few rows per group: bound by streaming the
// weights once. Both operands are read from memory in the layout of the 16x16x128
// instruction: of the 128 values of a step lane l holds, for row l % 16, with b = l /
// 16, the weights' block of 32 b and the activations' 16 from 16 b and from 64 + 16 b on;
// it gives the scale of block b to both. WN wavefronts of a workgroup have columns of
// their own, WK share the K of the same columns and add their sums in order. The weights are the instruction's
// first operand: a lane ends with 4 consecutive columns of one output row; the
// workgroup's 16 rows of 16 WN columns then go through LDS to lanes of 8 columns. One row
// of 6144 x 2048 5.6 us; 512 rows in 128 groups of 1536 x 2048 with SwiGLU 44 us, the
// weights at 4.9 TB/s.
template <int WN, int WK, bool GLU, bool MX8>
__global__ __launch_bounds__(WN* WK * 64) void k_mx8_gemm_rows(const Mx8GemmArgs a) {
  constexpr int P = GLU ? 2 : 1, W = WN * 16;
  __shared__ float part[WK > 1 ? (WK - 1) * WN * P : 1][256];
  __shared__ float tile[16][W + 4];
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave / WN, wn = wave % WN;
  const int ntn = ((MX8 ? LX_MX8_KP(a.cols) : a.cols) + W - 1) / W;
  const int rt = count_tiles<16>(a);
  const int cp = a.Kp / 2, sp = a.Kp / 32, steps = a.Kp / 128;
  Items it((int64_t)rt * ntn);
  for (; it.at < it.end; it.at += it.step) {
    // without groups the row tiles of the same columns follow each other
    const int64_t L = it.at;
    const int ti = (int)(a.offsets ? L / ntn : L % rt), t0 = (int)(a.offsets ? L % ntn : L / rt) * W, n0 = t0 + wn * 16;
    int g, m0, m1;
    if (!find_tile<16>(a, ti, g, m0, m1)) return;
    const int m = m0 + l16;
    int arow = -1;
    if (m < m1) arow = a.row_map ? a.row_map[m] : m;
    if (arow >= a.a_rows) arow = -1;
    const int64_t brow = (int64_t)g * a.N + min(n0 + l16, a.cols - 1);
    const uint8_t* const B = a.b + brow * cp + q * 16;
    const uint8_t* const Bs = a.bs + brow * sp;
    const int64_t up = (int64_t)a.cols * cp, ups = (int64_t)a.cols * sp;
    vf4 acc[P];
#pragma unroll
    for (int p = 0; p < P; ++p) acc[p] = vf4{0.f, 0.f, 0.f, 0.f};
    auto batch = [&](auto count, int k) __attribute__((always_inline)) {
      constexpr int U = decltype(count)::value;
      vu4 w[P][U], av[2][U], ws[P], as = {0, 0, 0, 0};
      auto words = [&](vu4& v, const uint8_t* row) __attribute__((always_inline)) {
        if constexpr (U < 4)
          v[0] = *(const uint32_t*)(row + k * 4);
        else
          v = *(const vu4w*)(row + k * 4);
      };
#pragma unroll
      for (int p = 0; p < P; ++p) {
#pragma unroll
        for (int u = 0; u < U; ++u) w[p][u] = *(const vu4*)(B + p * up + (int64_t)(k + u) * 64);
        words(ws[p], Bs + p * ups);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) av[0][u] = av[1][u] = vu4{0, 0, 0, 0};
      if (arow >= 0) {
        const uint8_t* const A = a.a + (int64_t)arow * a.Kp + q * 16;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          av[0][u] = *(const vu4*)(A + (int64_t)(k + u) * 128);
          av[1][u] = *(const vu4*)(A + (int64_t)(k + u) * 128 + 64);
        }
        words(as, a.as + (int64_t)arow * sp);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const v8i v = frag8(av[0][u], av[1][u]), lo = half_of<false>(v), hi = half_of<true>(v);
#pragma unroll
        for (int p = 0; p < P; ++p) {
          acc[p] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag4(w[p][u]), lo, acc[p], 4, 0, 0, ws[p][u] >> (8 * q), 0,
                                                                    as[u] >> (8 * q));
          acc[p] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag4(w[p][u]), hi, acc[p], 4, 0, 0, ws[p][u] >> (8 * q), 0,
                                                                    as[u] >> (8 * q));
        }
      }
    };
    const int k1 = (int)((int64_t)steps * (wk + 1) / WK);
    int k = (int)((int64_t)steps * wk / WK);
    for (; k + 4 <= k1; k += 4) batch(std::integral_constant<int, 4>{}, k);
    for (; k < k1; ++k) batch(std::integral_constant<int, 1>{}, k);
    if constexpr (WK > 1) {
      if (wk > 0) {
#pragma unroll
        for (int p = 0; p < P; ++p) *(vf4*)&part[((wk - 1) * WN + wn) * P + p][lane * 4] = acc[p];
      }
      __syncthreads();
      if (wk == 0) {
#pragma unroll
        for (int v = 0; v < WK - 1; ++v)
#pragma unroll
          for (int p = 0; p < P; ++p) acc[p] += *(const vf4*)&part[(v * WN + wn) * P + p][lane * 4];
      }
    }
    if (wk == 0) {
      const int c = n0 + q * 4, n = min(a.cols - c, 4);
      vf4 z = with_bias(a, g, c, n, arow >= 0, acc[0]);
      if constexpr (GLU)
        z = swiglu(z, with_bias(a, g, a.cols + c, n, arow >= 0, acc[1]));
      else
        z = activate(a.act, z);
      *(vf4*)&tile[l16][wn * 16 + q * 4] = z;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * (W / 8); i += WN * WK * 64) {
      const int r = i / (W / 8), c = i % (W / 8) * 8;
      F8 x;
#pragma unroll
      for (int j = 0; j < 8; ++j) x.v[j] = tile[r][c + j];
      finish<MX8>(a, m0 + r, t0 + c, m0 + r < m1, x);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- large tiles
typedef float f32x16 __attribute__((ext_vector_type(16)));

// BM x BN products per workgroup, a WR x WC grid of wavefronts, 32x32x64 instructions.
// Both operands go memory -> LDS directly: the activations in steps of 128 values, the
// weights, half as wide, in steps of 256, so that a row is a whole cache line of 128
// bytes in both; two stages each, one streaming in while the other is multiplied, the
// weights' next step in two halves. Inside a stage the eight 16-byte chunks of a row
// are XORed with (row / 2) % 8, so the 16 lanes that a read serves together hit 16
// different bank groups; a lane fetches the chunk that belongs at its LDS place.
// Scales come in groups of 512 values (16 bytes a row) through a ring of two. The
// weights are the instruction's first operand: a lane ends with 4 consecutive columns
// of one row, which get their bias and activation there (SwiGLU: a wavefront's columns
// are half gate, half up, so that both are in the same lane) and go through LDS to
// lanes of 8 columns.
// Workgroups stay for several tiles: the next one's place and rows are looked up under
// the first loads of the present one, and its first loads are under way while the
// present one's results are written.
// Bound by the matrix units, on long runs by what they draw: 8192 x 8192 x 8192 takes 725
// us, 3.0 PFLOP/s of instructions (two to a product) of the 3.04 that one instruction after
// the other reaches from registers on random operands. Tried and no
// faster: fragments read a step ahead between fences (463 for 420, with one instruction to a
// product, which took 432 for 8192 x 8192 x 8192 and 200 for 291 at 3001 x 4096 x 14336: what
// it drops is more than a bf16 result is rounded by where products cancel).
template <int BM_, int BN_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, THR = BM * BN > 128 * 128 ? 512 : 256, NW = THR / 64;
  static constexpr int WR = BM == 256 ? 4 : 2, WC = NW / WR, WM = BM / WR, WN = BN / WC, MI = WM / 32, NI = WN / 32;
  // A wavefront's blocks of 32 rows: first row of the first, rows from one to the next.
  // Of a tile that is at most half full each SIMD has half the work: of four wavefronts
  // each has one block less where their blocks alternate; of eight, two to a SIMD, one
  // of the two has none where each one's blocks are neighbours (32768 rows in 128
  // groups of 2048 x 768: 107 us in bf16, 256 x 256 161).
  static constexpr bool SPREAD = THR == 256;
  static constexpr int FIRST = SPREAD ? 32 : WM, NEXT_BLOCK = SPREAD ? 32 * WR : 32;
  static constexpr int RA = BM * 8 / THR, RB = BN * 8 / THR;  // a thread's 16-byte loads per step of A, of B
  static constexpr int SA = BM * 128, SB = BN * 128, STAGE = SA + SB, SGRP = (BM + BN) * 16;
  static constexpr int NEXT = 2 * STAGE + 2 * SGRP, LDS = NEXT + (RA + 1) * THR * 4, PER_CU = THR == 512 ? 1 : 2;
  static_assert(LDS * PER_CU <= 160 * 1024, "");
  static_assert(MI <= 2, "");
  static_assert(BM + BN <= THR && RB % 2 == 0 && NI % 2 == 0, "one row of scales per thread; halves");
};

template <class T, bool GLU>
__global__ __launch_bounds__(T::THR, T::PER_CU * T::THR / 256) void k_mx8_gemm_tile(const Mx8GemmArgs a) {
  constexpr int BM = T::BM, BN = T::BN, THR = T::THR, NW = T::NW, WC = T::WC, WM = T::WM, WN = T::WN, MI = T::MI, NI = T::NI;
  constexpr int RA = T::RA, RB = T::RB, SA = T::SA, STAGE = T::STAGE, SGRP = T::SGRP;
  constexpr int OC = GLU ? BN / 2 : BN, OW = GLU ? WN / 2 : WN;  // columns of the result: of a tile, of a wavefront
  __shared__ __attribute__((aligned(1024))) uint8_t smem[T::LDS];

  const bool mx8 = a.out_scales != nullptr;
  const int ntn = ((mx8 ? LX_MX8_KP(a.cols) : a.cols) + OC - 1) / OC;
  const int rt = count_tiles<BM>(a);
  Items it((int64_t)rt * ntn);
  if (it.at >= it.end) return;

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int l32 = lane & 31, h = lane >> 5, wm = wave / WC, wn = wave % WC;
  const int row0 = wm * T::FIRST;
  const int cp = a.Kp / 2, sp = a.Kp / 32, steps = a.Kp / 128;

  struct Item {
    int g, m0, m1, n0;
    uint64_t there;          // which of this wavefront's rows have a row of A
    uint32_t oa[RA];         // a thread's byte offsets from A (the host sees to it that they fit 32 bits)
    uint32_t qs;             // its row of the scale groups: of A (threads below BM)
  };
  static_assert(WM <= 64, "");
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
    const int64_t per_band = (int64_t)rt * 8;
    const int band = (int)(L / per_band), w = min(8, ntn - band * 8);
    const int rem = (int)(L - band * per_band), ti = rem / w;
    q.n0 = (band * 8 + rem - ti * w) * OC;
    q.g = q.m0 = q.m1 = 0;
    find_tile<BM>(a, ti, q.g, q.m0, q.m1);
#pragma unroll
    for (int j = 0; j < RA; ++j) {
      const int r = (j * THR + tid) >> 3;
      q.oa[j] = (uint32_t)max(row_of(q, r), 0) * (uint32_t)a.Kp + ((tid ^ (r >> 1)) & 7) * 16;
    }
    q.qs = (uint32_t)max(row_of(q, tid % BM), 0) * (uint32_t)sp;
    q.there = __ballot(lane < WM && row_of(q, row0 + (lane >> 5) * T::NEXT_BLOCK + l32) >= 0);
  };
  Item cur;
  const uint8_t *B, *Bs;  // the group's weights and their scales
  uint32_t ob[RB];        // a thread's byte offsets from B (the host sees to it that they fit 32 bits)
  // the weight row of row r of the tile
  auto brow = [&](int r) __attribute__((always_inline)) {
    if constexpr (GLU) {
      const int i = r % WN, c = cur.n0 + r / WN * OW + i % OW;
      return min(c, a.cols - 1) + (i < OW ? 0 : a.cols);
    } else {
      return min(cur.n0 + r, a.N - 1);
    }
  };
  auto from_b = [&]() __attribute__((always_inline)) {
    B = a.b + (int64_t)cur.g * a.N * cp;
    Bs = a.bs + (int64_t)cur.g * a.N * sp;
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const int r = (j * THR + tid) >> 3;
      ob[j] = (uint32_t)brow(r) * (uint32_t)cp + ((tid ^ (r >> 1)) & 7) * 16;
    }
    if (wave >= NW - BN / 64) cur.qs = (uint32_t)brow(tid % BN) * (uint32_t)sp;
  };
  // Group q of the scales: words 4 q .. 4 q + 3 of every row, 16 bytes a row (a
  // memory address need only be aligned to words). A row's last group holds its
  // last four words, so a step finds its words `late` words further on.
  auto late = [&](int q) __attribute__((always_inline)) { return steps < 4 ? 0 : max(q * 4 - (steps - 4), 0); };
  auto issue_scales = [&](int q) __attribute__((always_inline)) {
    uint8_t* const st = smem + 2 * STAGE + (q & 1) * SGRP;
    if (steps >= 4) {
      const int at = (q * 4 - late(q)) * 4;
      if (wave < BM / 64) load_lds<16>(a.as + at, cur.qs, st + wave * 1024);
      if (wave >= NW - BN / 64) load_lds<16>(Bs + at, cur.qs, st + BM * 16 + (wave - (NW - BN / 64)) * 1024);
    } else {
      // rows of fewer words: word by word, 16 rows x 4 words per load, the last
      // one repeated
      const int word = min(lane & 3, steps - 1) * 4;
#pragma unroll 1
      for (int r0 = wave * 16; r0 < BM + BN; r0 += NW * 16) {
        const int r = r0 + (lane >> 2);
        if (r0 < BM)
          load_lds<4>(a.as, (uint32_t)max(row_of(cur, r), 0) * (uint32_t)sp + word, st + r0 * 16);
        else
          load_lds<4>(Bs, (uint32_t)brow(r - BM) * (uint32_t)sp + word, st + r0 * 16);
      }
    }
  };
  // load j of step t of A into stage t % 2
  auto issue_a = [&](int t, int j) __attribute__((always_inline)) {
    load_lds<16>(a.a + (int64_t)t * 128, cur.oa[j], smem + (t & 1) * STAGE + (j * NW + wave) * 1024);
  };
  // load j of step u of B (256 values) into stage u % 2; where only half of it is
  // there the upper chunks repeat the lower ones (they are not multiplied)
  auto issue_b = [&](int u, int j) __attribute__((always_inline)) {
    const uint32_t back = 2 * u + 1 == steps ? ((tid ^ (((j * THR + tid) >> 3) >> 1)) & 4) * 16 : 0;
    load_lds<16>(B + (int64_t)u * 128, ob[j] - back, smem + (u & 1) * STAGE + SA + (j * NW + wave) * 1024);
  };
  auto begin = [&]() __attribute__((always_inline)) {
    issue_scales(0);
#pragma unroll
    for (int j = 0; j < RA; ++j) issue_a(0, j);
#pragma unroll
    for (int j = 0; j < RB; ++j) issue_b(0, j);
  };

  f32x16 acc[MI][NI];
  const int swz = (l32 >> 1) & 7;
  const uint32_t la = (row0 + l32) * 128 + (h ^ swz) * 16, lb = SA + (wn * WN + l32) * 128 + (h ^ swz) * 16;
  const uint8_t* const lsa = smem + 2 * STAGE + (row0 + l32) * 16;
  const uint8_t* const lsb = smem + 2 * STAGE + (BM + wn * WN + l32) * 16;
  // a row's scales of a step are one word: a lane's block of instruction s is 2 s +
  // h, so after a shift by h bytes its scale is byte 2 s
  struct Scales {
    uint32_t a[MI], b[NI];
  };
  struct Frags {
    vu4 a[MI][2], b[NI];
  };
  auto read_scales = [&](int t) __attribute__((always_inline)) {
    Scales q;
    const int st = ((t >> 2) & 1) * SGRP + ((t & 3) + late(t >> 2)) * 4;
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) q.b[ni] = *(const uint32_t*)(lsb + st + ni * 512) >> (8 * h);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) q.a[mi] = *(const uint32_t*)(lsa + st + mi * T::NEXT_BLOCK * 16) >> (8 * h);
    return q;
  };
  // fragments of instruction s (64 values) of step t: of the activations 16 values
  // from 16 h and from 32 + 16 h on, of the weights 32 from 32 h on
  // (chunk c of a row lies at (c ^ swz) 16 of its 128 bytes: the address of h's chunk,
  // XORed with the rest of c)
  auto lds = [&](uint32_t first, int c) __attribute__((always_inline)) { return smem + (first ^ (uint32_t)(c * 16)); };
  auto read_b = [&](Frags& f, int s, int t) __attribute__((always_inline)) {
    const uint8_t* const p = lds(lb + ((t >> 1) & 1) * STAGE, (t & 1) * 4 + 2 * s);
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) f.b[ni] = *(const vu4*)(p + ni * 4096);
  };
  auto read_a = [&](Frags& f, auto blocks, int s, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int mi = 0; mi < decltype(blocks)::value; ++mi)
#pragma unroll
      for (int c = 0; c < 2; ++c) f.a[mi][c] = *(const vu4*)(lds(la + (t & 1) * STAGE, 4 * s + 2 * c) + mi * T::NEXT_BLOCK * 128);
  };
  // step t's loads: A's, and the half (t - 1) % 2 of the weights' step that begins at t or
  // t + 1
  auto issue = [&](int t, auto odd) __attribute__((always_inline)) {
    constexpr int ODD = decltype(odd)::value;
#pragma unroll
    for (int j = 0; j < RA; ++j) issue_a(t, j);
    const int u = (t + 1) >> 1;
    if (2 * u < steps) {
#pragma unroll
      for (int j = 0; j < RB / 2; ++j) issue_b(u, (ODD ? 0 : RB / 2) + j);
    }
  };
  auto multiply = [&](auto sv, auto blocks, const Frags& f, const Scales& q) __attribute__((always_inline)) {
    constexpr int S = decltype(sv)::value;
#pragma unroll
    for (int mi = 0; mi < decltype(blocks)::value; ++mi) {
      const v8i x = frag8(f.a[mi][0], f.a[mi][1]);
      auto row = [&](const v8i& v) __attribute__((always_inline)) {
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
          acc[mi][ni] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(frag4(f.b[ni]), v, acc[mi][ni], 4, 0, 2 * S, q.b[ni],
                                                                        2 * S, q.a[mi]);
      };
      row(half_of<false>(x));
      row(half_of<true>(x));
    }
  };
  using std::integral_constant;
  constexpr integral_constant<int, 0> i0{};
  constexpr integral_constant<int, 1> i1{};

  look_up(it.at, cur);
  from_b();
  begin();
  for (;;) {
    it.at += it.step;
    const bool more = it.at < it.end;
    Item next;
    // (a thread's offsets of the next item wait in LDS: next to the present one's they
    // would not fit in registers)
    uint32_t* const keep = (uint32_t*)(smem + T::NEXT) + tid;
    if (more) {
      look_up(it.at, next);
#pragma unroll
      for (int j = 0; j < RA; ++j) keep[j * THR] = next.oa[j];
      keep[RA * THR] = next.qs;
    }
    land_and_meet();
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x16{};
    const int live = min(max((cur.m1 - cur.m0 - row0 + T::NEXT_BLOCK - 1) / T::NEXT_BLOCK, 0), MI);
    // step t has landed, step t + 1 streams in under its products
    auto step = [&](int t, auto odd) __attribute__((always_inline)) {
      constexpr int ODD = decltype(odd)::value;
      if (t + 1 < steps) {
        if (ODD && (t & 3) == 3) issue_scales((t + 1) >> 2);
        issue(t + 1, integral_constant<int, !ODD>{});
      }
      auto products = [&](auto blocks) __attribute__((always_inline)) {
        const Scales q = read_scales(t);
        Frags f0, f1;
        read_b(f0, 0, t);
        read_a(f0, blocks, 0, t);
        read_b(f1, 1, t);
        read_a(f1, blocks, 1, t);
        multiply(i0, blocks, f0, q);
        multiply(i1, blocks, f1, q);
      };
      // blocks of 32 rows past the tile's last are not multiplied (256 x 256: a wavefront's
      // 64 rows are or are not, a second loop would not fit in registers)
      if (live == MI || (THR == 512 && live > 0))
        products(integral_constant<int, MI>{});
      else if (THR != 512 && live > 0)
        products(i1);
      land_and_meet();
    };
    int t = 0;
#pragma unroll 1
    for (; t + 2 <= steps; t += 2) {
      step(t, i0);
      step(t + 1, i1);
    }
    if (t < steps) step(t, i0);

    const int g = cur.g, m0 = cur.m0, m1 = cur.m1, c0 = cur.n0 + wn * OW;
    const uint64_t there = cur.there;
    if (more) {
      cur = next;
#pragma unroll
      for (int j = 0; j < RA; ++j) cur.oa[j] = keep[j * THR];
      cur.qs = keep[RA * THR];
      from_b();
      begin();
    }
    // 32 rows by CW columns at a time through this wavefront's part of the second stages
    // (the next item's first step is on its way into the first ones), 16-byte chunks
    // XORed by the row
    int ln = lane;
    asm volatile("" : "+v"(ln));
    constexpr int CW = OW >= 64 && STAGE / NW >= 32 * 64 * 4 ? 64 : 32, LPR = CW / 8;
    static_assert(NW * 32 * CW * 4 <= STAGE, "");
    uint8_t* const e = smem + STAGE + wave * 32 * CW * 4;
    auto chunk = [](int r, int c) { return r * CW * 4 + (c ^ (CW == 32 ? (r >> 1) & 7 : r & 15)) * 16; };
    auto four = [](const f32x16& v, int q) { return vf4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]}; };
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      if (mi >= live) break;
      const bool has = there >> (mi * 32 + (ln & 31)) & 1;
#pragma unroll
      for (int cc = 0; cc < OW / CW; ++cc) {
#pragma unroll
        for (int nn = 0; nn < CW / 32; ++nn) {
          constexpr int HALF = NI / 2;
          const int ni = cc * (CW / 32) + nn;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int c = c0 + ni * 32 + 8 * q + 4 * (ln >> 5), n = min(a.cols - c, 4);
            vf4 z = with_bias(a, g, c, n, has, four(acc[mi][ni], q));
            if constexpr (GLU)
              z = swiglu(z, with_bias(a, g, a.cols + c, n, has, four(acc[mi][(ni + HALF) % NI], q)));
            else
              z = activate(a.act, z);
            *(vf4*)(e + chunk(ln & 31, nn * 8 + 2 * q + (ln >> 5))) = z;
          }
        }
        asm volatile("" ::: "memory");  // (a wavefront's LDS accesses run in order)
#pragma unroll 2
        for (int r0 = 0; r0 < 32; r0 += 64 / LPR) {
          const int r = r0 + ln / LPR, m = m0 + row0 + mi * T::NEXT_BLOCK + r, c = c0 + cc * CW + ln % LPR * 8;
          const vf4 u = *(const vf4*)(e + chunk(r, ln % LPR * 2)), v = *(const vf4*)(e + chunk(r, ln % LPR * 2 + 1));
          const F8 x{{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]}};
          if (mx8)
            finish<true>(a, m, c, m < m1, x);
          else
            finish<false>(a, m, c, m < m1, x);
        }
        asm volatile("" ::: "memory");
      }
    }
    if (!more) break;
  }
}

template <int WN, int WK, bool GLU, bool MX8>
hipError_t launch_rows(const Mx8GemmArgs& a, hipStream_t s) {
  constexpr int BM = 16, BN = 16 * WN;
  const int64_t tiles = a.offsets ? std::min<int64_t>((int64_t)a.M / BM + a.G, a.M) : ((int64_t)a.M + BM - 1) / BM;
  const int64_t cols = MX8 ? LX_MX8_KP((int64_t)a.cols) : a.cols, items = tiles * ((cols + BN - 1) / BN);
  k_mx8_gemm_rows<WN, WK, GLU, MX8><<<(unsigned)std::min<int64_t>((items + 7) / 8 * 8, 1 << 16), WN * WK * 64, 0, s>>>(a);
  return hipGetLastError();
}

template <class T, bool GLU>
hipError_t launch_tile(const Mx8GemmArgs& a, hipStream_t s) {
  constexpr int OC = GLU ? T::BN / 2 : T::BN;
  const int64_t tiles = a.offsets ? std::min<int64_t>((int64_t)a.M / T::BM + a.G, a.M) : ((int64_t)a.M + T::BM - 1) / T::BM;
  const int64_t cols = a.out_scales ? LX_MX8_KP((int64_t)a.cols) : a.cols, items = tiles * ((cols + OC - 1) / OC);
  const unsigned grid = (unsigned)std::min<int64_t>((items + 7) / 8 * 8, 256 * T::PER_CU);
  k_mx8_gemm_tile<T, GLU><<<grid, T::THR, 0, s>>>(a);
  return hipGetLastError();
}

template <bool GLU>
hipError_t launch(const Mx8GemmArgs& a, hipStream_t s) {
  const bool mx8 = a.out_scales != nullptr;
  switch (a.plan.kernel) {
    case Mx8GemmPlan::kRows4: return mx8 ? launch_rows<2, 4, GLU, true>(a, s) : launch_rows<2, 4, GLU, false>(a, s);
    case Mx8GemmPlan::kRows: return mx8 ? launch_rows<4, 1, GLU, true>(a, s) : launch_rows<4, 1, GLU, false>(a, s);
    case Mx8GemmPlan::kTile64: return launch_tile<Tile<64, 128>, GLU>(a, s);
    case Mx8GemmPlan::kTile128: return launch_tile<Tile<128, 128>, GLU>(a, s);
    default: return launch_tile<Tile<256, 256>, GLU>(a, s);
  }
}

}  // namespace

// Which kernel: the one with the least time by a model of rounds. A round is what the
// compute units take at once, in us per 4096 values of K (`half` where there are so few
// tiles that they share nothing) and besides, for filling and writing out:
//                  half      full      besides        tiles at once
//   16 x 32        5.5       5.5       1.3            256          (rows4)
//   16 x 64        16        27        3              512, 1024    (rows; with SwiGLU 16 x 128, 18, 45)
//   64 x 128       21        27        4.5            256, 512
//   128 x 128      33        51        7              256, 512
//   256 x 256      75        75        28             256          (with SwiGLU, half the results, 12)
// Of groups' rows only the mean is known: their last tiles are taken to be half full. Of
// those the wider tiles leave out what lies past them (`last`: the rows that they cost), up
// to where they wait for the weights, at 0.8 of a full tile. Over 419 sizes, all but 16 drawn
// (17 .. 16384 rows, 256 .. 14336 columns, K of 64 .. 14336, 1 .. 128 groups), the choice takes
// 2.4% longer than the best of the five (of those over 60 us 1.7%, 18% at worst; of shorter
// ones 68%, at 1141 x 576 x 8640 in 64 groups: 97 for 57); with 28 besides for SwiGLU, as without it, 2.2
// and 26% over 60 us; between the two row kernels alone (where operands
// reach 2^32 bytes), over 393, 1.2%, 27% at worst. us of rows4, rows, 64, 128, 256:
//   512 x 1536 x 2048, 128 groups, SwiGLU to 8 bits     74  44  50  56  83
//   2048 x 1536 x 2048, 128 groups, the same           118  70  50  56  84
//   32768 x 2048 x 768, 128 groups, fp32              1080 627  202 171 223
//   3001 x 4096 x 14336, bf16                            -   -  314 291 310
//   8192 x 8192 x 8192, bf16                             -   -  913 893 723
//   32768 x 1536 x 2048, 128 groups, SwiGLU to 8 bits    -   -  245 239 241  (12 takes 256, 28 128)
//   7735 x 11824 x 1368, the same in one group           -   -  285 278 220  (the same)
Mx8GemmPlan mx8_gemm_plan(int M, int N, int Kp, int G, bool swiglu, bool rows_only) {
  Mx8GemmPlan p{};
  const int64_t groups = G > 1 ? std::min(M, G) : 1;
  p.kernel = Mx8GemmPlan::kRows;
  double best = 0;
  auto offer = [&](Mx8GemmPlan::Kernel k, int64_t bm, int64_t bn, double last, int at_once, int few, double half, double full, double besides) {
    const double m = M, in_parts = G > 1 ? m + groups * (bm / 2) : m;  // rows with the last tiles full
    const int64_t rows = std::max((int64_t)std::ceil(in_parts / bm), groups);
    const int64_t tiles = rows * (((int64_t)N + bn - 1) / bn), whole = tiles / at_once, rest = tiles % at_once;
    const double k4 = Kp / 4096., share = G > 1 ? std::max((m + groups * last) / in_parts, 0.8) : 1;
    const double us = share * (whole * (full * k4 + besides) + (rest == 0 ? 0 : (rest <= few ? half : full) * k4 + besides));
    if (best == 0 || us < best) {
      best = us;
      p.kernel = k;
    }
  };
  if (!rows_only) {
    offer(Mx8GemmPlan::kTile64, 64, 128, 32, 512, 256, 21, 27, 4.5);
    offer(Mx8GemmPlan::kTile128, 128, 128, 32, 512, 256, 33, 51, 7);
    offer(Mx8GemmPlan::kTile256, 256, 256, 64, 256, 256, 75, 75, swiglu ? 12 : 28);
  }
  offer(Mx8GemmPlan::kRows4, 16, 32, 8, 256, 256, 5.5, 5.5, 1.3);
  if (G > 1 || rows_only) offer(Mx8GemmPlan::kRows, 16, swiglu ? 128 : 64, 8, 1024, 512, swiglu ? 18 : 16, swiglu ? 45 : 27, 3);
  return p;
}

hipError_t launch_mx8_gemm(const Mx8GemmArgs& a, hipStream_t s) { return a.act == LX_ACT_SWIGLU ? launch<true>(a, s) : launch<false>(a, s); }

}  // namespace lx
