// Microscaled 8-bit values: rounding and reading back (layout and rules in
// lorex_block.h).
#include "lx_block.h"
#include "lx_mx8.h"
#include "lx_rowwise.h"

namespace lx {
namespace {

// Both directions are bound by memory, but for SwiGLU's exponential and quotient. A
// lane has 8 values of a row, 4 lanes share a block of 32; rows as in the 4-bit
// rounding. Rounding 3001 x 14336 in bf16 27 us (130 MB, 4.9 TB/s), 8192 x 4096 22 to 24, 4096 x
// 4096 9; with SwiGLU 3001 x 14336 in bf16 64 (216 MB, 3.4 TB/s), 32768 x 768 53 (2.4), in
// fp32 46 (5.0); reading 8192 x 4096 back 16.4 (102 MB, 6.2 TB/s, in part from cache).
template <int U, bool SWIGLU>
__global__ __launch_bounds__(256) void k_mx8_quantize(const Mx4Args a, int tpr) {
  const int Kp = LX_MX8_KP(a.K);
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
      const uint2 code = mx8_round(x, s);
      if (row < a.rows) {
        *(uint2*)(a.codes + row * Kp + c) = code;
        if ((c & 31) == 0) a.scales[row * (Kp / 32) + c / 32] = (uint8_t)s;
      }
    }
  });
}

template <int U>
__global__ __launch_bounds__(256) void k_mx8_dequantize(const Mx4Args a, int tpr) {
  const int Kp = LX_MX8_KP(a.K);
  for_rows<U>(a.rows, a.K / 8, tpr, [&](int64_t r, int rpb, int c) {
    uint2 code[U];
    uint32_t s[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t row = r + (int64_t)j * rpb;
      code[j] = make_uint2(0, 0);
      s[j] = 0;
      if (row < a.rows) {
        code[j] = *(const uint2*)(a.codes + row * Kp + c);
        s[j] = a.scales[row * (Kp / 32) + c / 32];
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t row = r + (int64_t)j * rpb;
      const float f = mx_scale(s[j]);
      F8 x;
      auto two = [&](uint32_t w, auto hi, float& p, float& q) {
        const auto v = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, decltype(hi)::value);
        p = v[0] * f;
        q = v[1] * f;
      };
      two(code[j].x, std::false_type{}, x.v[0], x.v[1]);
      two(code[j].x, std::true_type{}, x.v[2], x.v[3]);
      two(code[j].y, std::false_type{}, x.v[4], x.v[5]);
      two(code[j].y, std::true_type{}, x.v[6], x.v[7]);
      if (row < a.rows) store8((void*)a.x, a.f32, row * a.K + c, x);
    }
  });
}

}  // namespace

hipError_t launch_mx8_quantize(const Mx4Args& a, hipStream_t s) {
  const int tpr = row_lanes(LX_MX8_KP(a.K) / 8);
  const bool many = row_grid(a.rows, tpr, 4) >= 2048;
  const int grid = row_grid(a.rows, tpr, many ? 4 : 1);
  if (a.swiglu)
    many ? k_mx8_quantize<4, true><<<grid, 256, 0, s>>>(a, tpr) : k_mx8_quantize<1, true><<<grid, 256, 0, s>>>(a, tpr);
  else
    many ? k_mx8_quantize<4, false><<<grid, 256, 0, s>>>(a, tpr) : k_mx8_quantize<1, false><<<grid, 256, 0, s>>>(a, tpr);
  return hipGetLastError();
}

hipError_t launch_mx8_dequantize(const Mx4Args& a, hipStream_t s) {
  const int tpr = row_lanes(a.K / 8);
  const bool many = row_grid(a.rows, tpr, 4) >= 2048;
  const int grid = row_grid(a.rows, tpr, many ? 4 : 1);
  many ? k_mx8_dequantize<4><<<grid, 256, 0, s>>>(a, tpr) : k_mx8_dequantize<1><<<grid, 256, 0, s>>>(a, tpr);
  return hipGetLastError();
}

}  // namespace lx
