// Rows of the block norms: sums over a row's lanes, and the forward (formulas in
// lorex_block.h), for kernels that differ in what they do with the next block's
// input. Included after lx_block.h.
#pragma once

#include <type_traits>

#include "lx_philox.h"
#include "lx_vec.h"

namespace lx {

// Sums of N values over the TPR lanes of a row. With more than one wavefront
// per row each call takes LDS slots of its own (`lds`, N per wavefront of the
// workgroup), so that one barrier per call is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float* lds) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = lane_sum<64>(x[i]);
  if constexpr (TPR > 64) {
    constexpr int NW = TPR / 64;
    const int wave = threadIdx.x >> 6, w0 = wave / NW * NW;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) lds[wave * N + i] = x[i];
    }
    __syncthreads();
    // each lane takes one wavefront's sum
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lds[(w0 + threadIdx.x % NW) * N + i];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lane_sum<NW>(x[i]);
  }
}

__device__ __forceinline__ float rms(float sum, int d, float eps) { return 1.f / sqrtf(sum / (float)d + eps); }

// Forward workgroups: 256 threads, or one row's if it needs more.
template <int TPR>
constexpr int kFwdThreads = TPR < 256 ? 256 : TPR;

// One workgroup's rows. put(t, column, whether the column exists, whether the row
// does, 8 values) is called by all lanes; lds: 2 floats per wavefront. DROP: the
// block's output is dropped out. LEAN: h, y and
// the weights are bf16 and there are no slots, which leaves room in registers for all
// the wavefronts that a compute unit can hold.
template <int TPR, int NV, bool DROP, bool LEAN, class Put>
__device__ __forceinline__ void block_norm_rows(const NormArgs& a, float* lds, Put&& put) {
  constexpr int RPB = kFwdThreads<TPR> / TPR, NW = kFwdThreads<TPR> / 64;
  using Raw = std::conditional_t<LEAN, RawB8, Raw8>;
  const bool slots = !LEAN && a.slot_row;
  const bool h_f32 = !LEAN && a.h_f32, y_f32 = !LEAN && a.y_f32, w_f32 = !LEAN && a.w_f32;
  DropoutKeys keys{};
  if constexpr (DROP) keys = dropout_keys(a.drop);
  const int lt = threadIdx.x % TPR;
  int col[NV];
  bool in[NV];
  F8 sw[NV], wp[NV];  // scale w_post; w_pre
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    col[i] = (i * TPR + lt) * 8;
    in[i] = col[i] < a.d;
    sw[i] = wp[i] = F8{{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}};
    if (in[i]) {
      if (a.w_pre) wp[i] = load8(a.w_pre, w_f32, col[i]);
      if (a.w_post) sw[i] = load8(a.w_post, w_f32, col[i]);
      if (a.scale) {
        const F8 q = load8(a.scale, w_f32, col[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sw[i].v[e] *= q.v[e];
      }
    }
  }
  // (all rows of the workgroup run as many rounds: the barriers need them. The
  // row's index stays one value per lane: uniform, the slots' loads go through the
  // scalar cache, and one token's 8 slots at d = 1024 take 4.7 us for 4.3)
  const int g = (int)threadIdx.x / TPR;
  for (int64_t t0 = (int64_t)blockIdx.x * RPB; t0 < a.T; t0 += (int64_t)gridDim.x * RPB) {
    const int64_t t = t0 + g;
    const bool live = RPB == 1 || t < a.T;
    const int64_t row = t * a.d;
    Raw rh[NV], ry[NV];
    F8 h[NV], y[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      rh[i] = ry[i] = Raw{};
      if (in[i] && live) {
        rh[i] = load_as<Raw>(a.h, h_f32, row + col[i]);
        if (a.y && !slots) ry[i] = load_as<Raw>(a.y, y_f32, row + col[i]);
      }
    }
    if (a.y) {
      const float gate = a.gate && live ? a.gate[t] : 1.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) y[i] = slots ? F8{} : unpack8(ry[i], y_f32);
      if (slots && a.y_rows > 0 && live) {
        // four slots' rows at a time; a dropped slot reads row 0 and adds nothing
        for (int j0 = 0; j0 < a.k; j0 += 4) {
          int r[4];
          float w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            r[j] = j0 + j < a.k ? a.slot_row[t * a.k + j0 + j] : -1;
            w[j] = j0 + j < a.k ? a.slot_weights[t * a.k + j0 + j] : 0.f;
            if (r[j] >= a.y_rows) r[j] = -1;
          }
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            Raw q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              q[j] = Raw{};
              if (in[i]) q[j] = load_as<Raw>(a.y, y_f32, (int64_t)max(r[j], 0) * a.d + col[i]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (r[j] >= 0) {
                const F8 v = unpack8(q[j], y_f32);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[i].v[e] += w[j] * v.v[e];
              }
          }
        }
      }
      float f = DROP ? a.drop.scale : gate;  // with dropout the gate comes after it
      if (a.w_post) {
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) s[0] += y[i].v[e] * y[i].v[e];
        row_sums<TPR>(s, lds);
        f *= rms(s[0], a.d, a.eps);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        h[i] = unpack8(rh[i], h_f32);
        if constexpr (DROP) {
          // (a dropped value adds 0 even where the row's factor or a weight is not finite)
          const uint32_t kept = dropout_kept(a.drop, keys, col[i] / 8, (uint32_t)t);
#pragma unroll
          for (int e = 0; e < 8; ++e) h[i].v[e] = a.alpha * h[i].v[e] + gate * (kept >> e & 1 ? f * y[i].v[e] * sw[i].v[e] : 0.f);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) h[i].v[e] = a.alpha * h[i].v[e] + f * (y[i].v[e] * sw[i].v[e]);
        }
        if (in[i] && live) store8(a.h_out, h_f32, row + col[i], h[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) h[i] = unpack8(rh[i], h_f32);
    }
    if (a.w_pre) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += in[i] ? h[i].v[e] * h[i].v[e] : 0.f;
      row_sums<TPR>(s, lds + NW);
      const float r = rms(s[0], a.d, a.eps);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        F8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x.v[e] = h[i].v[e] * r * wp[i].v[e];
        put(t, col[i], in[i], live, x);
      }
    }
    // without both sums a row has one barrier or none: the next row may only
    // write the slots when all have read them
    if constexpr (TPR > 64)
      if (!(a.y && a.w_post && a.w_pre)) __syncthreads();
  }
}

}  // namespace lx
