// Products of 8-bit activations and 4-bit weights per group of rows, with bias,
// activation and residual (formulas and layout in lorex_block.h), on the
// block-scaled matrix instructions with one operand e2m1 and the other e4m3.
#include "lx_block.h"
#include "lx_groups.h"
#include "lx_mx8.h"
#include "lx_vec.h"

#include <algorithm>
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
// its bits are lost then (the sums of normal values are off by 1e-5 of their size;
// with both operands e2m1 nothing is). Activations whose exponent field's top bit is
// set (from 2 on under the block's scale) and the others are within the window among
// themselves, so two instructions, one for each, drop nothing.
struct Halves {
  v8i hi, lo;
};
__device__ __forceinline__ Halves halves(const v8i& a) {
  Halves r;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t m = ((uint32_t)a[j] >> 6) & 0x01010101u, mask = (m << 8) - m;
    r.hi[j] = a[j] & (int)mask;
    r.lo[j] = a[j] & (int)~mask;
  }
  return r;
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
    if (act == LX_ACT_SILU) z[j] = z[j] / (1.f + expf(-z[j]));
    if (act == LX_ACT_GELU) z[j] = 0.5f * z[j] * erfcf(z[j] * -0.70710678118654752f);
  }
  return z;
}
__device__ __forceinline__ vf4 swiglu(vf4 z, vf4 u) {
#pragma unroll
  for (int j = 0; j < 4; ++j) z[j] = z[j] / (1.f + expf(-z[j])) * u[j];
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
// it gives the scale of block b to both. WN wavefronts of a workgroup have columns of their own, WK share the K of
// the same columns and add their sums in order. The weights are the instruction's
// first operand: a lane ends with 4 consecutive columns of one output row; the
// workgroup's 16 rows of 16 WN columns then go through LDS to lanes of 8 columns.
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
        const Halves v = halves(frag8(av[0][u], av[1][u]));
#pragma unroll
        for (int p = 0; p < P; ++p) {
          acc[p] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag4(w[p][u]), v.lo, acc[p], 4, 0, 0, ws[p][u] >> (8 * q), 0,
                                                                    as[u] >> (8 * q));
          acc[p] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag4(w[p][u]), v.hi, acc[p], 4, 0, 0, ws[p][u] >> (8 * q), 0,
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

template <int WN, int WK, bool GLU, bool MX8>
hipError_t launch_rows(const Mx8GemmArgs& a, hipStream_t s) {
  constexpr int BM = 16, BN = 16 * WN;
  const int64_t tiles = a.offsets ? std::min<int64_t>((int64_t)a.M / BM + a.G, a.M) : ((int64_t)a.M + BM - 1) / BM;
  const int64_t cols = MX8 ? LX_MX8_KP((int64_t)a.cols) : a.cols, items = tiles * ((cols + BN - 1) / BN);
  k_mx8_gemm_rows<WN, WK, GLU, MX8><<<(unsigned)std::min<int64_t>((items + 7) / 8 * 8, 1 << 16), WN * WK * 64, 0, s>>>(a);
  return hipGetLastError();
}

template <bool GLU, bool MX8>
hipError_t launch(const Mx8GemmArgs& a, hipStream_t s) {
  switch (a.plan.kernel) {
    case Mx8GemmPlan::kRows4: return launch_rows<2, 4, GLU, MX8>(a, s);
    default: return launch_rows<4, 1, GLU, MX8>(a, s);
  }
}

}  // namespace

// Which kernel. Rows of a group are not known here, only their mean.
Mx8GemmPlan mx8_gemm_plan(int M, int cols, int Kp, int G) {
  Mx8GemmPlan p{};
  const int64_t waves = ((int64_t)cols + 15) / 16 * std::min(M, G);
  p.kernel = M <= 16 && waves <= 1024 ? Mx8GemmPlan::kRows4 : Mx8GemmPlan::kRows;
  return p;
}

hipError_t launch_mx8_gemm(const Mx8GemmArgs& a, hipStream_t s) {
  const bool mx8 = a.out_scales != nullptr;
  if (a.act == LX_ACT_SWIGLU) return mx8 ? launch<true, true>(a, s) : launch<true, false>(a, s);
  return mx8 ? launch<false, true>(a, s) : launch<false, false>(a, s);
}

}  // namespace lx
