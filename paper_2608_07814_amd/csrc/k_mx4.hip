// Microscaled 4-bit values (OCP MXFP4): rounding, reading back, and grouped
// products on the block-scaled matrix instructions (layout and rules in
// lorex_block.h).
#include "lx_block.h"
#include "lx_vec.h"

#include <algorithm>

namespace lx {
namespace {

constexpr int kBlk = 32;  // values under one scale

// ---------------------------------------------------------------- rounding
// A lane rounds 8 values, 4 lanes share a block of 32. The largest magnitude
// goes over the 4 lanes as bits: as unsigned integers magnitudes keep their
// order, and infinities and NaNs come out above every finite one. The
// conversion instruction divides by a power of two, rounds to nearest even and
// saturates at 6.
__global__ __launch_bounds__(256) void k_mx4_quantize(const Mx4Args a) {
  const int Kp = LX_MX4_KP(a.K);
  const int64_t n = a.rows * (Kp / 8);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / (Kp / 8);
    const int c = (int)(i - row * (Kp / 8)) * 8;
    F8 x = F8{};
    if (c < a.K) {
      if (a.swiglu) {
        const F8 g = load8(a.x, a.f32, row * 2 * a.K + c), u = load8(a.x, a.f32, row * 2 * a.K + a.K + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) x.v[e] = g.v[e] / (1.f + expf(-g.v[e])) * u.v[e];
      } else {
        x = load8(a.x, a.f32, row * a.K + c);
      }
    }
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x.v[e]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true));
    const int e = (int)(top >> 23);                  // biased; 255: infinity or NaN
    const bool bad = e == 255;
    const int s = bad ? 255 : e > 2 ? e - 2 : 0;     // scale byte
    uint32_t code = 0;
    if (!bad) {
      // (2^-127 is not a normal number: there the values are doubled instead)
      const float f = __uint_as_float((uint32_t)(s > 0 ? s : 1) << 23);
#pragma unroll
      for (int j = 0; j < 8; ++j) x.v[j] = s > 0 ? x.v[j] : 2.f * x.v[j];
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x.v[0], x.v[1], f, 0);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x.v[2], x.v[3], f, 1);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x.v[4], x.v[5], f, 2);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x.v[6], x.v[7], f, 3);
    }
    *(uint32_t*)(a.codes + row * (Kp / 2) + c / 2) = code;
    if ((c & (kBlk - 1)) == 0) a.scales[row * (Kp / kBlk) + c / kBlk] = (uint8_t)s;
  }
}

// 0.5 * the e2m1 value of a code, as an integer in half units: 0 1 2 3 4 6 8 12
__device__ __forceinline__ float mx4_value(uint32_t c) {
  const uint32_t m = c & 7;
  const float v = (float)(m < 4 ? m : m < 6 ? 2 * m - 4 : 4 * m - 16) * 0.5f;
  return c & 8 ? -v : v;
}

__global__ __launch_bounds__(256) void k_mx4_dequantize(const Mx4Args a) {
  const int Kp = LX_MX4_KP(a.K);
  const int64_t n = a.rows * (a.K / 8);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / (a.K / 8);
    const int c = (int)(i - row * (a.K / 8)) * 8;
    const uint32_t code = *(const uint32_t*)(a.codes + row * (Kp / 2) + c / 2);
    const int s = a.scales[row * (Kp / kBlk) + c / kBlk];
    F8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = s == 255 ? NAN : ldexpf(mx4_value(code >> (4 * e)), s - 127);
    store8((void*)a.x, a.f32, row * a.K + c, x);
  }
}

// ---------------------------------------------------------------- products
typedef int v8i __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v8i frag(const uint4& q) { return v8i{(int)q.x, (int)q.y, (int)q.z, (int)q.w, 0, 0, 0, 0}; }

// The group and the first row of row tile `tile` (tiles of BM rows, counted
// group by group), found by each wavefront: 64 groups at a time, a prefix sum
// of their tile counts over the lanes. false: there is no such tile.
template <int BM>
__device__ __forceinline__ bool find_tile(const Mx4GemmArgs& a, int tile, int& g, int& m0, int& m1) {
  if (!a.offsets) {
    g = 0;
    m0 = tile * BM;
    m1 = min(m0 + BM, a.M);
    return m0 < a.M;
  }
  const int lane = threadIdx.x & 63;
  for (int g0 = 0; g0 < a.G; g0 += 64) {
    int lo = 0, hi = 0;
    if (g0 + lane < a.G) {
      lo = min(max(a.offsets[g0 + lane], 0), a.M);
      hi = min(max(a.offsets[g0 + lane + 1], lo), a.M);
    }
    const int n = (hi - lo + BM - 1) / BM;
    int sum = n;  // inclusive prefix sum
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int q = __shfl_up(sum, o);
      if (lane >= o) sum += q;
    }
    const int all = __shfl(sum, 63);
    if (tile < all) {
      const int src = __builtin_ctzll(__ballot(tile < sum));
      g = g0 + src;
      const int first = __shfl(lo, src), last = __shfl(hi, src), before = __shfl(sum - n, src);
      m0 = first + (tile - before) * BM;
      m1 = min(m0 + BM, last);
      return true;
    }
    tile -= all;
  }
  return false;
}

// 16 rows x 64 columns per workgroup, 16 columns per wavefront, both operands
// read from memory in the layout of the 16x16x128 instruction: lane l holds
// row l % 16's block l / 16 of the 128 values of a step. The weights are the
// instruction's first operand, so a lane ends with 4 consecutive columns of
// one output row.
__global__ __launch_bounds__(256) void k_mx4_gemm(const Mx4GemmArgs a) {
  int g, m0, m1;
  if (!find_tile<16>(a, blockIdx.x, g, m0, m1)) return;
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
  const int n0 = blockIdx.y * 64 + (threadIdx.x >> 6) * 16;
  if (n0 >= a.N) return;
  const int m = m0 + l16;
  int ar = -1;
  if (m < m1) ar = a.row_map ? a.row_map[m] : m;
  const bool live = ar >= 0 && ar < a.a_rows;
  const int64_t arow = live ? ar : 0, brow = (int64_t)g * a.N + min(n0 + l16, a.N - 1);
  const int cp = a.Kp / 2, sp = a.Kp / 32;
  vf4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < a.Kp / 128; ++k) {
    uint4 av = make_uint4(0, 0, 0, 0);
    int as = 0;
    if (live) {
      av = *(const uint4*)(a.a + arow * cp + k * 64 + q * 16);
      as = a.as[arow * sp + k * 4 + q];
    }
    const uint4 bv = *(const uint4*)(a.b + brow * cp + k * 64 + q * 16);
    const int bs = a.bs[brow * sp + k * 4 + q];
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag(bv), frag(av), acc, 4, 4, 0, bs, 0, as);
  }
  if (m >= m1) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = n0 + q * 4 + i;
    if (n < a.N) {
      const int64_t at = (int64_t)m * a.N + n;
      if (a.out_f32)
        ((float*)a.out)[at] = acc[i];
      else
        ((uint16_t*)a.out)[at] = (uint16_t)pack_bf16(acc[i], 0.f);
    }
  }
}

}  // namespace

hipError_t launch_mx4_quantize(const Mx4Args& a, hipStream_t s) {
  const int64_t n = a.rows * (LX_MX4_KP(a.K) / 8);
  k_mx4_quantize<<<(int)std::min<int64_t>((n + 255) / 256, 1 << 16), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const Mx4Args& a, hipStream_t s) {
  const int64_t n = a.rows * (a.K / 8);
  k_mx4_dequantize<<<(int)std::min<int64_t>((n + 255) / 256, 1 << 16), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_mx4_gemm(const Mx4GemmArgs& a, hipStream_t s) {
  const int tiles = a.offsets ? (int)std::min<int64_t>((int64_t)a.M / 16 + a.G, a.M) : (a.M + 15) / 16;
  k_mx4_gemm<<<dim3(tiles, (a.N + 63) / 64), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lx
