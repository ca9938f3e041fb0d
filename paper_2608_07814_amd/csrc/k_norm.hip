// Block norms: the RMS norms before and after a block with its gate and
// residual scale, forward and backward (formulas in lorex_block.h).
//
// A token's row stays in the registers of the TPR lanes that own it (NV groups
// of 8 columns each), so every row is read once and written once; the row sums
// go over lanes by DPP, over wavefronts through LDS.
#include "lx_block.h"
#include "lx_vec.h"

#include <algorithm>

namespace lx {
namespace {

// Sums of N values over the TPR lanes of a row. With more than one wavefront
// per row each call takes LDS slots of its own (`slot`), so that one barrier
// per call is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float* lds, int slot) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = lane_sum<64>(x[i]);
  if constexpr (TPR > 64) {
    constexpr int NW = TPR / 64;
    float* s = lds + slot * NW * N;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[(threadIdx.x >> 6) * N + i] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) t += s[w * N + i];
      x[i] = t;
    }
  }
}

template <int TPR, int NV>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_block_norm(const NormArgs a) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
  __shared__ float lds[2 * (TPR / 64)];
  const int lt = threadIdx.x % TPR;
  const int t = blockIdx.x * RPB + (int)threadIdx.x / TPR;
  if (t >= a.T) return;  // (TPR > 64: one row per workgroup, so no barrier is missed)
  const int64_t row = (int64_t)t * a.d;
  F8 h[NV];
  bool in[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + lt) * 8;
    in[i] = c < a.d;
    if (in[i])
      h[i] = load8(a.h, a.h_f32, row + c);
    else
      h[i] = F8{};
  }
  if (a.y) {
    F8 y[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) y[i] = F8{};
    if (a.slot_row) {
      for (int j = 0; j < a.k; ++j) {
        const int r = a.slot_row[(int64_t)t * a.k + j];
        const float w = a.slot_weights[(int64_t)t * a.k + j];
        if (r < 0 || r >= a.y_rows) continue;
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (in[i]) {
            const F8 q = load8(a.y, a.y_f32, (int64_t)r * a.d + (i * TPR + lt) * 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[i].v[e] += w * q.v[e];
          }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (in[i]) y[i] = load8(a.y, a.y_f32, row + (i * TPR + lt) * 8);
    }
    float r = a.gate ? a.gate[t] : 1.f;
    if (a.w_post) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += y[i].v[e] * y[i].v[e];
      row_sums<TPR>(s, lds, 0);
      r *= 1.f / sqrtf(s[0] / (float)a.d + a.eps);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (in[i]) {
        const int c = (i * TPR + lt) * 8;
        if (a.w_post) {
          const F8 w = load8(a.w_post, a.w_f32, c);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[i].v[e] *= w.v[e];
        }
        if (a.scale) {
          const F8 w = load8(a.scale, a.w_f32, c);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[i].v[e] *= w.v[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i].v[e] = a.alpha * h[i].v[e] + r * y[i].v[e];
        store8(a.h_out, a.h_f32, row + c, h[i]);
      }
  }
  if (!a.w_pre) return;
  float s[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) s[0] += h[i].v[e] * h[i].v[e];
  row_sums<TPR>(s, lds, 1);
  const float r = 1.f / sqrtf(s[0] / (float)a.d + a.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (in[i]) {
      const int c = (i * TPR + lt) * 8;
      const F8 w = load8(a.w_pre, a.w_f32, c);
      F8 x;
#pragma unroll
      for (int e = 0; e < 8; ++e) x.v[e] = h[i].v[e] * r * w.v[e];
      store8(a.x, a.x_f32, row + c, x);
    }
}

// Backward. With m = h' r_h, n = y r_y (no w_post: n = y, r_y = 1), D the
// gradient of h':
//   D    = dh' + r_h (dx w_pre - m mean(dx w_pre m))
//   z    = sum_c D scale w_post n          (= dgate; gate z = sum_c dn n)
//   dy   = r_y gate (D scale w_post - n z / d)     (no w_post: gate D scale)
// so the row sums are {h'^2, y^2, dx w_pre h'} and then z. A row group keeps
// its sums of dx m (dw_pre) and of gate D n (dw_post = scale q, dscale =
// w_post q) in registers over its tokens and leaves them in part.
template <int TPR, int NV>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_block_norm_grad(const NormGradArgs a) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
  __shared__ float lds[2 * 4 * (TPR / 64)];
  const int lt = threadIdx.x % TPR;
  const int grp = blockIdx.x * RPB + (int)threadIdx.x / TPR;
  if (grp >= a.groups) return;
  F8 sp[NV], sq[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) sp[i] = sq[i] = F8{};
  for (int64_t t = grp; t < a.T; t += a.groups) {
    const int64_t row = t * a.d;
    F8 m[NV], y[NV], D[NV], dx[NV];
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lt) * 8;
      m[i] = y[i] = D[i] = dx[i] = F8{};
      if (c < a.d) {
        m[i] = load8(a.h_out, a.h_f32, row + c);
        if (a.dh_out) D[i] = load8(a.dh_out, a.h_f32, row + c);
        if (a.y) y[i] = load8(a.y, a.y_f32, row + c);
        if (a.dx) {
          dx[i] = load8(a.dx, a.x_f32, row + c);
          const F8 w = load8(a.w_pre, a.w_f32, c);
#pragma unroll
          for (int e = 0; e < 8; ++e) s[2] += dx[i].v[e] * w.v[e] * m[i].v[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s[0] += m[i].v[e] * m[i].v[e];
          s[1] += y[i].v[e] * y[i].v[e];
        }
      }
    }
    row_sums<TPR>(s, lds, 0);
    const float inv_d = 1.f / (float)a.d;
    const float rh = 1.f / sqrtf(s[0] * inv_d + a.eps);
    const float ry = a.w_post ? 1.f / sqrtf(s[1] * inv_d + a.eps) : 1.f;
    const float mean = rh * s[2] * inv_d;
    const float gate = a.gate ? a.gate[t] : 1.f;
    const float alpha = a.y ? a.alpha : 1.f;
    float z[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lt) * 8;
      if (c < a.d) {
        if (a.dx) {
          const F8 w = load8(a.w_pre, a.w_f32, c);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float mm = m[i].v[e] * rh;
            D[i].v[e] += rh * (dx[i].v[e] * w.v[e] - mm * mean);
            sp[i].v[e] += dx[i].v[e] * mm;
          }
        }
        F8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o.v[e] = alpha * D[i].v[e];
        store8(a.dh, a.h_f32, row + c, o);
        if (a.y) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            y[i].v[e] *= ry;
            sq[i].v[e] += gate * D[i].v[e] * y[i].v[e];
          }
          if (a.scale) {
            const F8 w = load8(a.scale, a.w_f32, c);
#pragma unroll
            for (int e = 0; e < 8; ++e) D[i].v[e] *= w.v[e];
          }
          if (a.w_post) {
            const F8 w = load8(a.w_post, a.w_f32, c);
#pragma unroll
            for (int e = 0; e < 8; ++e) D[i].v[e] *= w.v[e];
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) z[0] += D[i].v[e] * y[i].v[e];
        }
      }
    }
    if (!a.y) {
      if constexpr (TPR > 64) __syncthreads();  // the sums' slots are free again
      continue;
    }
    // (the next row's first sums reuse the slots that every wavefront has read
    // before this call's barrier)
    row_sums<TPR>(z, lds, 3);
    if (a.dgate && lt == 0) a.dgate[t] = z[0];
    const float zn = a.w_post ? z[0] * inv_d : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lt) * 8;
      if (c < a.d) {
        F8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o.v[e] = ry * gate * (D[i].v[e] - y[i].v[e] * zn);
        store8(a.dy, a.y_f32, row + c, o);
      }
    }
  }
  float* const p = a.part + (int64_t)grp * 2 * a.d;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + lt) * 8;
    if (c < a.d) {
      store8(p, true, c, sp[i]);
      store8(p + a.d, true, c, sq[i]);
    }
  }
}

// Sums of the row groups' partials: 32 columns per workgroup, its 32 rows of
// lanes take every 32nd group, then LDS adds them in a fixed order.
__global__ __launch_bounds__(1024) void k_block_norm_grad_sum(const NormGradArgs a) {
  __shared__ float lds[32][33];
  const int x = threadIdx.x & 31, yy = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + x;  // [0, 2d)
  float s = 0.f;
  if (col < 2 * a.d)
    for (int g = yy; g < a.groups; g += 32) s += a.part[(int64_t)g * 2 * a.d + col];
  lds[yy][x] = s;
  __syncthreads();
  if (yy || col >= 2 * a.d) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) s += lds[i][x];
  if (col < a.d) {
    if (a.dw_pre) a.dw_pre[col] = s;
    return;
  }
  const int c = col - a.d;
  auto w1 = [&](const void* p) {
    return !p ? 1.f : a.w_f32 ? ((const float*)p)[c] : __uint_as_float((uint32_t)((const uint16_t*)p)[c] << 16);
  };
  if (a.dw_post) a.dw_post[c] = w1(a.scale) * s;
  if (a.dscale) a.dscale[c] = w1(a.w_post) * s;
}

template <class F>
hipError_t by_width(int d, F&& f) {
  using std::integral_constant;
  if (d <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (d <= 1024) return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (d <= 2048) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (d <= 4096) return f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (d <= 8192) return f(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  if (d <= 16384) return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

}  // namespace

hipError_t launch_block_norm(const NormArgs& a, hipStream_t s) {
  return by_width(a.d, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    k_block_norm<TPR, NV><<<(a.T + RPB - 1) / RPB, RPB * TPR, 0, s>>>(a);
    return hipGetLastError();
  });
}

int norm_grad_groups(int T, int) { return std::min(std::max(T, 1), 512); }

hipError_t launch_block_norm_grad(const NormGradArgs& a, hipStream_t s) {
  return by_width(a.d, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    k_block_norm_grad<TPR, NV><<<(a.groups + RPB - 1) / RPB, RPB * TPR, 0, s>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_block_norm_grad_sum(const NormGradArgs& a, hipStream_t s) {
  k_block_norm_grad_sum<<<(2 * a.d + 31) / 32, 1024, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lx
