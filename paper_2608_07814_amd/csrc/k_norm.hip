// Block norms: the RMS norms before and after a block with its gate and
// residual scale, forward and backward (formulas in lorex_block.h).
//
// Bound by memory: every row is read once and written once. A token's row stays
// in the registers of the TPR lanes that own it, NV groups of 8 columns each;
// row sums go over lanes by DPP, over wavefronts through LDS. Workgroups stay
// for many rows, so the weight vectors are read once per workgroup. Measured:
// forward 8192 x 4096 (fp32 output of the block, bf16 streams) 68 us, 4.9 TB/s; all
// in bf16 46 us (268 MB, 5.9 TB/s, in part from cache), with dropout 49; 4096 x 2048
// with 8 experts' fp32 rows combined 57 us (319 MB, in part from cache);
// backward 8192 x 4096 (fp32 stream) 126 us, 4.8 TB/s (with dropout 123 of 606 MB; all in
// bf16 77, with dropout 85: the generator's 20 wide products a group of 8 columns show
// where the row kernel is not waiting for memory); a large copy reaches 5.45.
#include "lx_block.h"
#include "lx_norm_rows.h"
#include "lx_vec.h"

#include <algorithm>
#include <cfloat>
#include <type_traits>

namespace lx {
namespace {

template <int TPR, int NV, bool DROP = false, bool LEAN = false>
__global__ __launch_bounds__(kFwdThreads<TPR>) void k_block_norm(const NormArgs a) {
  __shared__ float lds[2 * kFwdThreads<TPR> / 64];
  block_norm_rows<TPR, NV, DROP, LEAN>(a, lds, [&](int64_t t, int col, bool in, bool live, const F8& x) __attribute__((always_inline)) {
    if (in && live) store8(a.x, a.x_f32, t * a.d + col, x);
  });
}

// Backward. With m = h' r_h, n = y r_y (no w_post: n = y, r_y = 1), D the
// gradient of h' and s = scale w_post:
//   D    = dh' + r_h (dx w_pre - m mean(dx w_pre m))
//   z    = sum_c D s n                             (= dgate; gate z = sum_c dn n)
//   dy   = r_y gate (D s - n z / d)                (no w_post: gate D s)
// z is linear in D, so all sums are over what is stored, {h'^2, y^2, dx w_pre h',
// dh' s y, dx w_pre s y, h' s y}, and are joined at once: one pass for the sums,
// one for the results, one barrier per row (with z summed from D after the others
// 8192 x 4096 with fp32 streams took 130 us for 126, 2048 x 8192 in bf16 55 for
// 50). A workgroup takes one row or several at a time and stays for all of its
// rows, one workgroup per compute unit; loading the next row ahead of the sums
// gave 49 for 50 us at 2048 x 8192 and cost 22.6 for 20.3 at 5000 x 1024. The
// sums over tokens of dx m (dw_pre) and of gate D n (dw_post = scale q, dscale =
// w_post q) stay in registers, are joined over the workgroup's rows in LDS and
// left in part, one pair of vectors per workgroup. KEEP: the row stays in
// registers, as it is stored, between the passes (and the weights for all rows);
// else (rows of more than 8192, which do not fit) both are read again, from L2
// (1024 x 16384 in bf16 67 us, with the row kept and the weights read again 96).
constexpr int kBwd = 1024;
__device__ __forceinline__ void again(RawB8& r) { asm volatile("" : "+v"(r.a)); }
__device__ __forceinline__ void again(Raw8& r) { asm volatile("" : "+v"(r.a), "+v"(r.b)); }

template <bool BF, int TPR, int NV, bool KEEP, bool DROP = false>
__global__ __launch_bounds__(kBwd) void k_block_norm_grad(const NormGradArgs a) {
  constexpr int RPB = kBwd / TPR, NW = kBwd / 64;
  using Raw = std::conditional_t<BF, RawB8, Raw8>;
  __shared__ float lds[2 * 6 * NW];
  __shared__ float join[RPB > 1 ? 2 * RPB * TPR * NV * 8 : 1];
  const int lt = threadIdx.x % TPR, g = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  auto col = [&](int i) __attribute__((always_inline)) { return (i * TPR + lt) * 8; };
  struct Weights {
    F8 pre, s;
  };
  auto weights = [&](int i) __attribute__((always_inline)) {
    Weights w;
    w.pre = w.s = F8{{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}};
    if (col(i) < a.d) {
      if (a.w_pre) w.pre = load8(a.w_pre, a.w_f32, col(i));
      if (a.w_post) w.s = load8(a.w_post, a.w_f32, col(i));
      if (a.scale) {
        const F8 q = load8(a.scale, a.w_f32, col(i));
#pragma unroll
        for (int e = 0; e < 8; ++e) w.s.v[e] *= q.v[e];
      }
    }
    return w;
  };
  struct Row {
    Raw m, y, D, dx;
  };
  auto load = [&](int i, int64_t t) __attribute__((always_inline)) {
    Row r;
    r.m = r.y = r.D = r.dx = Raw{};
    if (col(i) < a.d && t < a.T) {
      const int64_t at = t * a.d + col(i);
      if (a.y) r.y = load_as<Raw>(a.y, a.y_f32, at);
      if (a.dx) {  // (without the second norm no gradient depends on h_out)
        r.m = load_as<Raw>(a.h_out, a.h_f32, at);
        r.dx = load_as<Raw>(a.dx, a.x_f32, at);
      }
      if (a.dh_out) r.D = load_as<Raw>(a.dh_out, a.h_f32, at);
    }
    return r;
  };
  DropoutKeys keys{};
  if constexpr (DROP) keys = dropout_keys(a.drop);
  F8 sp[NV], sq[NV];
  Weights w[KEEP ? NV : 1];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    sp[i] = sq[i] = F8{};
    if constexpr (KEEP) w[i] = weights(i);
  }
  const float inv_d = 1.f / (float)a.d, alpha = a.y ? a.alpha : 1.f;
  const int64_t stride = (int64_t)a.groups * RPB;
  int slots = 0;  // the sums' LDS slots of this row: the previous row's may still be read
  // (all rows of the workgroup run as many rounds: the barriers need them)
  for (int64_t t0 = (int64_t)blockIdx.x * RPB; t0 < a.T; t0 += stride, slots ^= 6 * NW) {
    const int64_t t = t0 + g, row = t * a.d;
    const bool live = t < a.T;
    // with dropout: the columns that are kept, formed as in the forward; a dropped
    // value's product with its weight counts as 0 whatever they hold
    auto mask = [&](int i) __attribute__((always_inline)) {
      if constexpr (DROP) return dropout_kept(a.drop, keys, col(i) / 8, (uint32_t)t);
      return 0u;
    };
    auto drop = [&](float v, float w, uint32_t kept, int e) __attribute__((always_inline)) {
      if constexpr (DROP) return kept >> e & 1 ? w * (v * a.drop.scale) : 0.f;
      return w * v;
    };
    float s[6] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto add = [&](const Row& q, const Weights& w, uint32_t kept) __attribute__((always_inline)) {
      const F8 m = unpack8(q.m, a.h_f32), y = unpack8(q.y, a.y_f32), D = unpack8(q.D, a.h_f32), dx = unpack8(q.dx, a.x_f32);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float dm = dx.v[e] * w.pre.v[e], sy = drop(y.v[e], w.s.v[e], kept, e);
        s[0] += m.v[e] * m.v[e];
        s[1] += y.v[e] * y.v[e];
        s[2] += dm * m.v[e];
        s[3] += D.v[e] * sy;
        s[4] += dm * sy;
        s[5] += m.v[e] * sy;
      }
    };
    uint32_t kept[KEEP ? NV : 1];
    Row q[KEEP ? NV : 1];
    if constexpr (KEEP) {
#pragma unroll
      for (int i = 0; i < NV; ++i) q[i] = load(i, t);
#pragma unroll
      for (int i = 0; i < NV; ++i) add(q[i], w[i], kept[i] = mask(i));
    } else {
#pragma unroll 1
      for (int i = 0; i < NV; ++i) add(load(i, t), weights(i), mask(i));
    }
    const float gate = a.gate && live ? a.gate[t] : 1.f;
    row_sums<TPR>(s, lds + slots);
    // (a row past T has zeros only, and with eps = 0 an infinite factor: 0 times
    // it must not reach the sums over tokens)
    const float rh = a.dx && live ? rms(s[0], a.d, a.eps) : 0.f;
    const float ry = a.w_post && live ? rms(s[1], a.d, a.eps) : 1.f;
    const float mean = rh * s[2] * inv_d;
    const float z = ry * (a.dx ? s[3] + rh * (s[4] - rh * mean * s[5]) : s[3]);
    const float zn = a.w_post ? z * inv_d : 0.f;
    if (a.dgate && lt == 0 && live) a.dgate[t] = z;
    // (the row is unpacked anew: next to its stored form it would not fit)
    if constexpr (KEEP) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        again(q[i].m);
        again(q[i].y);
        again(q[i].D);
        again(q[i].dx);
      }
    }
    auto give = [&](int i, const Row& q, const Weights& w, uint32_t kept) __attribute__((always_inline)) {
      const F8 m = unpack8(q.m, a.h_f32), y = unpack8(q.y, a.y_f32), D = unpack8(q.D, a.h_f32), dx = unpack8(q.dx, a.x_f32);
      F8 dh, dy;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float mm = m.v[e] * rh, n = y.v[e] * ry, d = D.v[e] + rh * (dx.v[e] * w.pre.v[e] - mm * mean);
        sp[i].v[e] += dx.v[e] * mm;
        sq[i].v[e] += gate * d * drop(n, 1.f, kept, e);
        dh.v[e] = alpha * d;
        // (without w_post zn is 0 and dy does not depend on y, which may be infinite or
        // NaN: its product with 0 must not count. With w_post zn is NaN then. A
        // choice by a.w_post took 71 for 62 us at 1024 x 16384)
        dy.v[e] = ry * gate * (d * drop(w.s.v[e], 1.f, kept, e) - __builtin_amdgcn_fmed3f(n, -FLT_MAX, FLT_MAX) * zn);
      }
      if (col(i) < a.d && live) {
        store8(a.dh, a.h_f32, row + col(i), dh);
        if (a.y) store8(a.dy, a.y_f32, row + col(i), dy);
      }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if constexpr (KEEP) {
        give(i, q[i], w[i], kept[i]);
      } else {
        asm volatile("" ::: "memory");  // (one group's loads at a time)
        give(i, load(i, t), weights(i), mask(i));
      }
    }
  }
  float* const p = a.part + (int64_t)blockIdx.x * 2 * a.d;
  if constexpr (RPB == 1) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (col(i) < a.d) {
        store8(p, true, col(i), sp[i]);
        store8(p + a.d, true, col(i), sq[i]);
      }
  } else {
    constexpr int W = TPR * NV * 8;  // columns of a row's lanes
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      store8(join + g * 2 * W, true, col(i), sp[i]);
      store8(join + g * 2 * W + W, true, col(i), sq[i]);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * W; c += kBwd) {
      float q = 0.f;
#pragma unroll
      for (int r = 0; r < RPB; ++r) q += join[r * 2 * W + c];
      const int e = c < W ? c : c - W;
      if (e < a.d) p[(c < W ? 0 : a.d) + e] = q;
    }
  }
}

// Sums of the workgroups' partials: 32 columns per workgroup, its 32 rows of
// lanes take every 32nd partial, then LDS adds them in a fixed order.
__global__ __launch_bounds__(1024) void k_block_norm_grad_sum(const NormGradArgs a) {
  __shared__ float lds[32][33];
  const int x = threadIdx.x & 31, yy = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + x;  // [0, 2d)
  float s = 0.f;
  if (col < 2 * a.d)
#pragma unroll 8
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
  // (no tokens, and with dropout a column that all of them drop, give 0 whatever the weights hold)
  const bool none = (a.drop.rng || a.T == 0) && s == 0.f;
  if (a.dw_post) a.dw_post[c] = none ? 0.f : w1(a.scale) * s;
  if (a.dscale) a.dscale[c] = none ? 0.f : w1(a.w_post) * s;
}

// Lanes of a row and groups of 8 columns per lane: a row's lanes hold one group
// each as long as 1024 lanes do.
template <class F>
hipError_t by_width(int d, F&& f) {
  using std::integral_constant;
#define LX_W(T, N) f(integral_constant<int, T>{}, integral_constant<int, N>{})
  if (d <= 512) return LX_W(64, 1);
  if (d <= 1024) return LX_W(128, 1);
  if (d <= 2048) return LX_W(256, 1);
  if (d <= 4096) return LX_W(512, 1);
  if (d <= 8192) return LX_W(1024, 1);
  if (d <= 16384) return LX_W(1024, 2);
  return LX_W(1024, 4);
#undef LX_W
}

}  // namespace

hipError_t launch_block_norm(const NormArgs& a, hipStream_t s) {
  return by_width(a.d, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, THR = kFwdThreads<TPR>;
    constexpr int RPB = THR / TPR;
    const int grid = (int)std::min<int64_t>(((int64_t)a.T + RPB - 1) / RPB, 256 * (2048 / THR));
    const bool lean = norm_lean(a);
    if (a.drop.rng)
      lean ? k_block_norm<TPR, NV, true, true><<<grid, THR, 0, s>>>(a) : k_block_norm<TPR, NV, true><<<grid, THR, 0, s>>>(a);
    else
      lean ? k_block_norm<TPR, NV, false, true><<<grid, THR, 0, s>>>(a) : k_block_norm<TPR, NV><<<grid, THR, 0, s>>>(a);
    return hipGetLastError();
  });
}

int norm_grad_groups(int T, int d) {
  int at_once = 1;
  (void)by_width(d, [&](auto tpr, auto) {
    at_once = kBwd / decltype(tpr)::value;
    return hipSuccess;
  });
  return (int)std::min<int64_t>(std::max<int64_t>(((int64_t)T + at_once - 1) / at_once, 1), 256);
}

hipError_t launch_block_norm_grad(const NormGradArgs& a, hipStream_t s) {
  const bool bf = !a.h_f32 && (!a.y || !a.y_f32) && (!a.dx || !a.x_f32);
  return by_width(a.d, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    auto go = [&](auto b, auto drop) {
      k_block_norm_grad<decltype(b)::value, TPR, NV, NV == 1, decltype(drop)::value><<<a.groups, kBwd, 0, s>>>(a);
    };
    if (a.drop.rng)
      bf ? go(std::true_type{}, std::true_type{}) : go(std::false_type{}, std::true_type{});
    else
      bf ? go(std::true_type{}, std::false_type{}) : go(std::false_type{}, std::false_type{});
    return hipGetLastError();
  });
}

hipError_t launch_block_norm_grad_sum(const NormGradArgs& a, hipStream_t s) {
  k_block_norm_grad_sum<<<(2 * a.d + 31) / 32, 1024, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lx
