// The router's load-balance loss and its gradient (formulas in lorex_block.h).
//
// LPT lanes own one token's row of logits and keep it in registers, lane l
// the columns VEC (l + LPT i) .. + VEC - 1 of chunk i, so each row is read once;
// maximum and sums go over those lanes by DPP. In the forward a lane adds up
// its columns' probabilities over its tokens; a workgroup joins its lane
// groups' sums in LDS in a fixed order, and a second launch joins the
// workgroups'.
#include "lx_block.h"
#include "lx_vec.h"

#include <algorithm>

namespace lx {
namespace {

constexpr int kThreads = 256;

template <int VEC>
struct Cols {
  float v[VEC];
};

template <int VEC>
__device__ __forceinline__ Cols<VEC> load_cols(const void* p, bool f32, int64_t i) {
  Cols<VEC> o;
  if constexpr (VEC == 8) {
    const F8 q = load8(p, f32, i);
#pragma unroll
    for (int e = 0; e < 8; ++e) o.v[e] = q.v[e];
  } else {
    o.v[0] = f32 ? ((const float*)p)[i] : __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
  }
  return o;
}

template <int VEC>
__device__ __forceinline__ void store_cols(void* p, bool f32, int64_t i, const Cols<VEC>& x) {
  if constexpr (VEC == 8) {
    F8 q;
#pragma unroll
    for (int e = 0; e < 8; ++e) q.v[e] = x.v[e];
    store8(p, f32, i, q);
  } else if (f32) {
    ((float*)p)[i] = x.v[0];
  } else {
    ((uint16_t*)p)[i] = (uint16_t)pack_bf16(x.v[0], 0.f);
  }
}

// The softmax of one row (lanes of masked or missing tokens: live = false,
// nothing is read and p = 0).
template <int VEC, int LPT, int NCH>
__device__ __forceinline__ void row_softmax(const void* logits, bool f32, int64_t row, int E, int l, bool live,
                                            Cols<VEC> (&p)[NCH]) {
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (i * LPT + l) * VEC;
    const bool in = live && c < E;
    if (in) p[i] = load_cols<VEC>(logits, f32, row + c);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if (!in) p[i].v[e] = -INFINITY;
      mx = fmaxf(mx, p[i].v[e]);  // (a NaN is dropped here and comes back through exp)
    }
  }
  mx = lane_max<LPT>(mx);
  const float base = mx == -INFINITY ? 0.f : mx;  // only -inf: every exp below is 0
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      p[i].v[e] = expf(p[i].v[e] - base);
      s += p[i].v[e];
    }
  s = lane_sum<LPT>(s);
  const float inv = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e) p[i].v[e] *= inv;
}

// loss, prob and n_tokens from the sums of one expert per thread in turn
__device__ __forceinline__ void finish(const BalanceArgs& a, const float* sum_p, const int32_t* counts, int n,
                                       float* red) {
  const float inv_n = n > 0 ? 1.f / (float)n : 0.f;
  float part = 0.f;
  for (int e = threadIdx.x; e < a.E; e += blockDim.x) {
    const float p = sum_p[e] * inv_n;
    a.prob[e] = p;
    a.counts[e] = counts[e];
    part += (float)counts[e] * p;
  }
  part = lane_sum<64>(part);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = part;
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.f;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) s += red[w];
    *a.loss = n > 0 ? a.coef * (float)a.E * (s * inv_n / (float)a.k) : 0.f;
    *a.n_tokens = n;
  }
}

template <int VEC, int LPT, int NCH>
__global__ __launch_bounds__(kThreads) void k_balance(const BalanceArgs a) {
  constexpr int TPB = kThreads / LPT;
  __shared__ float sp[kBalanceMaxE];
  __shared__ int32_t sc[kBalanceMaxE];
  __shared__ int32_t sn;
  __shared__ float red[kThreads / 64];
  const int l = threadIdx.x % LPT, g = threadIdx.x / LPT;
  for (int e = threadIdx.x; e < a.E; e += kThreads) {
    sp[e] = 0.f;
    sc[e] = 0;
  }
  if (threadIdx.x == 0) sn = 0;
  __syncthreads();
  Cols<VEC> acc[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[i].v[e] = 0.f;
  int n = 0;
  // (every lane of the workgroup runs as many rounds: the exchanges need them)
  for (int t0 = blockIdx.x * TPB; t0 < a.T; t0 += gridDim.x * TPB) {
    const int t = t0 + g;
    const bool live = t < a.T && (!a.mask || a.mask[t]);
    Cols<VEC> p[NCH];
    row_softmax<VEC, LPT, NCH>(a.logits, a.f32, (int64_t)t * a.E, a.E, l, live, p);
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[i].v[e] += p[i].v[e];
    if (live) {
      n += l == 0;
      for (int j = l; j < a.k; j += LPT) {
        const int id = a.ids[(int64_t)t * a.k + j];
        if (id >= 0 && id < a.E) atomicAdd(&sc[id], 1);
      }
    }
  }
  if (n) atomicAdd(&sn, n);
  // the lane groups add their sums one after the other
  for (int q = 0; q < TPB; ++q) {
    if (g == q) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = (i * LPT + l) * VEC;
        if (c < a.E)
#pragma unroll
          for (int e = 0; e < VEC; ++e) sp[c + e] += acc[i].v[e];
      }
    }
    __syncthreads();
  }
  if (gridDim.x == 1) {
    finish(a, sp, sc, sn, red);
    return;
  }
  const int64_t at = (int64_t)blockIdx.x * a.E;
  for (int e = threadIdx.x; e < a.E; e += kThreads) {
    a.part_p[at + e] = sp[e];
    a.part_c[at + e] = sc[e];
  }
  if (threadIdx.x == 0) a.part_n[blockIdx.x] = sn;
}

// The workgroups' sums, by one workgroup.
__global__ __launch_bounds__(1024) void k_balance_sum(const BalanceArgs a) {
  __shared__ float sp[1024];
  __shared__ int32_t sc[1024];
  __shared__ float red[16];
  __shared__ int32_t sn;
  if (threadIdx.x == 0) {
    int n = 0;
    for (int b = 0; b < a.blocks; ++b) n += a.part_n[b];
    sn = n;
  }
  for (int e = threadIdx.x; e < a.E; e += 1024) {
    float p = 0.f;
    int c = 0;
    for (int b = 0; b < a.blocks; ++b) {
      p += a.part_p[(int64_t)b * a.E + e];
      c += a.part_c[(int64_t)b * a.E + e];
    }
    sp[e] = p;
    sc[e] = c;
  }
  __syncthreads();
  finish(a, sp, sc, sn, red);
}

template <int VEC, int LPT, int NCH>
__global__ __launch_bounds__(kThreads) void k_balance_grad(const BalanceArgs a) {
  constexpr int TPB = kThreads / LPT;
  const int l = threadIdx.x % LPT, g = threadIdx.x / LPT;
  const int n = *a.n_tokens;
  const float inv_n = n > 0 ? 1.f / (float)n : 0.f;
  const float w = (a.dloss ? *a.dloss : 1.f) * a.coef * (float)a.E * inv_n * inv_n / (float)a.k;
  Cols<VEC> f[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (i * LPT + l) * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[i].v[e] = c < a.E ? (float)a.counts[c + e] : 0.f;
  }
  for (int t0 = blockIdx.x * TPB; t0 < a.T; t0 += gridDim.x * TPB) {
    const int t = t0 + g;
    const bool live = t < a.T && (!a.mask || a.mask[t]);
    const int64_t row = (int64_t)t * a.E;
    Cols<VEC> p[NCH];
    row_softmax<VEC, LPT, NCH>(a.logits, a.f32, row, a.E, l, live, p);
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) dot += p[i].v[e] * f[i].v[e];
    dot = lane_sum<LPT>(dot);
    if (t < a.T) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = (i * LPT + l) * VEC;
        if (c < a.E) {
          Cols<VEC> o;
#pragma unroll
          for (int e = 0; e < VEC; ++e) o.v[e] = live ? p[i].v[e] * w * (f[i].v[e] - dot) : 0.f;
          store_cols<VEC>(a.dlogits, a.f32, row + c, o);
        }
      }
    }
  }
}

// Rows of a multiple of 8 logits are read 16 bytes (bf16) at a time by as few
// lanes as hold the row, others one logit at a time.
template <class F>
hipError_t by_experts(int E, F&& f) {
  using std::integral_constant;
#define LX_E(V, L, N) f(integral_constant<int, V>{}, integral_constant<int, L>{}, integral_constant<int, N>{})
  if (E % 8 == 0) {
    if (E <= 64) return LX_E(8, 8, 1);
    if (E <= 128) return LX_E(8, 16, 1);
    if (E <= 256) return LX_E(8, 32, 1);
    if (E <= 512) return LX_E(8, 64, 1);
    return LX_E(8, 64, 2);
  }
  if (E <= 64) return LX_E(1, 64, 1);
  if (E <= 128) return LX_E(1, 64, 2);
  if (E <= 256) return LX_E(1, 64, 4);
  if (E <= 512) return LX_E(1, 64, 8);
  return LX_E(1, 64, 16);
#undef LX_E
}

int tokens_per_block(int E) {
  int tpb = 0;
  (void)by_experts(E, [&](auto, auto lpt, auto) {
    tpb = kThreads / decltype(lpt)::value;
    return hipSuccess;
  });
  return tpb;
}

}  // namespace

int balance_blocks(int T, int E) {
  const int tpb = tokens_per_block(E);
  return std::min(std::max((T + 4 * tpb - 1) / (4 * tpb), 1), 256);
}

hipError_t launch_balance(const BalanceArgs& a, hipStream_t s) {
  return by_experts(a.E, [&](auto v, auto l, auto n) {
    k_balance<decltype(v)::value, decltype(l)::value, decltype(n)::value><<<a.blocks, kThreads, 0, s>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_balance_sum(const BalanceArgs& a, hipStream_t s) {
  k_balance_sum<<<1, 1024, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_balance_grad(const BalanceArgs& a, hipStream_t s) {
  const int tpb = tokens_per_block(a.E);
  const int grid = std::min((int)(((int64_t)a.T + tpb - 1) / tpb), 2048);
  return by_experts(a.E, [&](auto v, auto l, auto n) {
    k_balance_grad<decltype(v)::value, decltype(l)::value, decltype(n)::value><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace lx
