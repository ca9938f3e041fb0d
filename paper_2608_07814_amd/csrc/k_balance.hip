// The router's load-balance loss and its gradient (formulas in lorex_block.h).
//
// LPT lanes own one token's row of logits and keep it in registers, lane l
// the columns VEC (l + LPT i) .. + VEC - 1 of chunk i, so each row is read once;
// maximum and sums go over those lanes by DPP. In the forward a lane adds up
// its columns' probabilities over its tokens; the sums of a wavefront's lane
// groups are joined over lanes, the wavefronts' in LDS, the workgroups' by a
// second launch, each in a fixed order. Counts are integer LDS atomics: exact
// in any order. Bound by latency: 16384 x 256 in bf16 takes 10.0 + 4.6 us forward
// and 7.8 us backward, of which moving the 8.4 MB of logits is 1.5 and 3.
#include "lx_block.h"
#include "lx_vec.h"

#include <algorithm>

namespace lx {
namespace {

constexpr int kThreads = 256;  // gradient
constexpr int kFwd = 1024;     // forward: few workgroups, whose sums are joined by one

template <int VEC>
struct Cols {
  float v[VEC];
};

// A lane's logits of one row as they lie in memory, so that several rows' loads
// and the masks can be under way together. A masked token's are loaded too but
// not used.
template <int VEC, int NCH>
struct RowRaw {
  Raw8 v[VEC == 8 ? NCH : 1];
  uint32_t w[VEC == 8 ? 1 : NCH];
};

template <int VEC, int LPT, int NCH>
__device__ __forceinline__ void load_row(const BalanceArgs& a, int64_t t, int l, RowRaw<VEC, NCH>& r) {
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (i * LPT + l) * VEC;
    const bool in = t < a.T && c < a.E;
    if constexpr (VEC == 8) {
      r.v[i] = Raw8{};
      if (in) r.v[i] = load_raw8(a.logits, a.f32, t * a.E + c);
    } else {
      r.w[i] = 0;
      if (in) r.w[i] = a.f32 ? ((const uint32_t*)a.logits)[t * a.E + c] : (uint32_t)((const uint16_t*)a.logits)[t * a.E + c] << 16;
    }
  }
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

// e^x for x <= 0 in fp32: the product with log2(e) is kept as a rounded value and
// its remainder, so the relative error stays within a few 2^-24 where the result is a
// normal number, x >= -87.3 (through the rounded product alone it grows to 100 times
// that at x = -80), at a third of expf's instructions, which bound these kernels.
// Below that the result is 0: the instruction gives no smaller numbers, and a
// probability under 2^-126 is the choice of a softmax whose sum is at least 1.
__device__ __forceinline__ float exp_down(float x) {
  constexpr float kLog2e = 1.44269504f, kLog2eLow = 1.92596299e-8f, kLn2 = 0.693147181f;
  const float t = x * kLog2e;
  const float lo = fmaf(x, kLog2eLow, fmaf(x, kLog2e, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return x < -150.f ? 0.f : fmaf(e, lo * kLn2, e);  // (there e^x has no fp32 value but 0)
}

// The softmax of one row; lanes of masked or missing tokens (live = false): p = 0.
template <int VEC, int LPT, int NCH>
__device__ __forceinline__ void row_softmax(const RowRaw<VEC, NCH>& r, bool f32, int E, int l, bool live, Cols<VEC> (&p)[NCH]) {
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const bool in = live && (i * LPT + l) * VEC < E;
    if constexpr (VEC == 8) {
      const F8 q = unpack8(r.v[i], f32);
#pragma unroll
      for (int e = 0; e < 8; ++e) p[i].v[e] = q.v[e];
    } else {
      p[i].v[0] = __uint_as_float(r.w[i]);
    }
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
      p[i].v[e] = exp_down(p[i].v[e] - base);
      s += p[i].v[e];
    }
  s = lane_sum<LPT>(s);
  const float inv = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e) p[i].v[e] *= inv;
}

// The outputs from every expert's sums, by a workgroup of kFwd threads:
// thread e has expert e's.
__device__ __forceinline__ void finish(const BalanceArgs& a, float sum_p, int32_t count, int n) {
  __shared__ float red[kFwd / 64];
  const int e = threadIdx.x;
  const float inv_n = n > 0 ? 1.f / (float)n : 0.f;
  float part = 0.f;
  if (e < a.E) {
    const float p = sum_p * inv_n;
    a.prob[e] = p;
    a.counts[e] = count;
    part = (float)count * p;
  }
  part = lane_sum<64>(part);
  if ((e & 63) == 0) red[e >> 6] = part;
  __syncthreads();
  if (e == 0) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kFwd / 64; ++w) s += red[w];
    *a.loss = n > 0 ? a.coef * (float)a.E * (s * inv_n / (float)a.k) : 0.f;
    *a.n_tokens = n;
  }
}
static_assert(kFwd >= kBalanceMaxE, "one thread per expert");

template <int VEC, int LPT, int NCH>
__global__ __launch_bounds__(kFwd) void k_balance(const BalanceArgs a) {
  constexpr int TPB = kFwd / LPT, NW = kFwd / 64, COLS = VEC * LPT * NCH;
  __shared__ float sp[NW][COLS];
  __shared__ int32_t sc[COLS];
  __shared__ int32_t sn;
  const int l = threadIdx.x % LPT, g = threadIdx.x / LPT, wave = threadIdx.x >> 6;
  for (int e = threadIdx.x; e < COLS; e += kFwd) sc[e] = 0;
  if (threadIdx.x == 0) sn = 0;
  __syncthreads();
  Cols<VEC> acc[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[i].v[e] = 0.f;
  int n = 0;
  // the next round's loads are under way while this one's sums are formed (every
  // lane of the workgroup runs as many rounds: the exchanges need them)
  RowRaw<VEC, NCH> next;
  uint32_t mask = 1;
  int id = -1;
  auto load = [&](int64_t t) __attribute__((always_inline)) {
    load_row<VEC, LPT, NCH>(a, t, l, next);
    mask = t < a.T ? a.mask ? a.mask[t] : 1 : 0;
    id = t < a.T && l < a.k ? a.ids[t * a.k + l] : -1;
  };
  const int64_t stride = (int64_t)gridDim.x * TPB;
  load((int64_t)blockIdx.x * TPB + g);
  for (int64_t t0 = (int64_t)blockIdx.x * TPB; t0 < a.T; t0 += stride) {
    const int64_t t = t0 + g;
    const RowRaw<VEC, NCH> row = next;
    const bool live = mask != 0;
    int first = id;
    if (t0 + stride < a.T) load(t + stride);
    Cols<VEC> p[NCH];
    row_softmax<VEC, LPT, NCH>(row, a.f32, a.E, l, live, p);
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[i].v[e] += p[i].v[e];
    if (live) {
      n += l == 0;
      if (first >= 0 && first < a.E) atomicAdd(&sc[first], 1);
      for (int j = l + LPT; j < a.k; j += LPT) {
        const int more = a.ids[t * a.k + j];
        if (more >= 0 && more < a.E) atomicAdd(&sc[more], 1);
      }
    }
  }
  if (n) atomicAdd(&sn, n);
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float s = stride_sum<LPT>(acc[i].v[e]);
      if ((threadIdx.x & 63) < LPT) sp[wave][(i * LPT + l) * VEC + e] = s;
    }
  __syncthreads();
  const int e = threadIdx.x;
  float s = 0.f;
  int32_t c = 0;
  if (e < a.E) {
#pragma unroll
    for (int w = 0; w < NW; ++w) s += sp[w][e];
    c = sc[e];
  }
  if (gridDim.x == 1) {
    finish(a, s, c, sn);
    return;
  }
  if (e < a.E) {
    a.part_p[(int64_t)blockIdx.x * a.E + e] = s;
    a.part_c[(int64_t)blockIdx.x * a.E + e] = c;
  }
  if (e == 0) a.part_n[blockIdx.x] = sn;
}

// The workgroups' sums, by one workgroup: thread (expert, slice) takes every
// S-th workgroup's, then the slices are joined in order.
__global__ __launch_bounds__(kFwd) void k_balance_sum(const BalanceArgs a) {
  __shared__ float sp[kFwd];
  __shared__ int32_t sc[kFwd];
  __shared__ int32_t sn;
  const int S = kFwd / a.E, e = threadIdx.x % a.E, q = threadIdx.x / a.E;
  if (threadIdx.x < 64) {
    int n = 0;
    for (int b = threadIdx.x; b < a.blocks; b += 64) n += a.part_n[b];
#pragma unroll
    for (int o = 32; o; o >>= 1) n += __shfl_xor(n, o);
    if (threadIdx.x == 0) sn = n;
  }
  float p = 0.f;
  int32_t c = 0;
  if (q < S) {
#pragma unroll 8
    for (int b = q; b < a.blocks; b += S) {
      p += a.part_p[(int64_t)b * a.E + e];
      c += a.part_c[(int64_t)b * a.E + e];
    }
  }
  sp[threadIdx.x] = p;
  sc[threadIdx.x] = c;
  __syncthreads();
  if (q == 0)
    for (int i = 1; i < S; ++i) {
      p += sp[i * a.E + e];
      c += sc[i * a.E + e];
    }
  finish(a, p, c, sn);
}

template <int VEC, int LPT, int NCH>
__global__ __launch_bounds__(kThreads) void k_balance_grad(const BalanceArgs a) {
  constexpr int TPB = kThreads / LPT;
  const int l = threadIdx.x % LPT, g = threadIdx.x / LPT;
  const int64_t stride = (int64_t)gridDim.x * TPB;
  RowRaw<VEC, NCH> next;
  uint32_t mask = 1;
  auto load = [&](int64_t t) __attribute__((always_inline)) {
    load_row<VEC, LPT, NCH>(a, t, l, next);
    mask = t < a.T ? a.mask ? a.mask[t] : 1 : 0;
  };
  load((int64_t)blockIdx.x * TPB + g);
  // the counts go through LDS: read by every wavefront from memory, their few
  // cache lines held the launch up (16384 x 256: 10.8 against 7.8 us)
  __shared__ float counts[VEC * LPT * NCH];
  for (int e = threadIdx.x; e < VEC * LPT * NCH; e += kThreads) counts[e] = e < a.E ? (float)a.counts[e] : 0.f;
  __syncthreads();
  Cols<VEC> f[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[i].v[e] = counts[(i * LPT + l) * VEC + e];
  const int n = *a.n_tokens;
  const float inv_n = n > 0 ? 1.f / (float)n : 0.f;
  const float w = (a.dloss ? *a.dloss : 1.f) * a.coef * (float)a.E * inv_n * inv_n / (float)a.k;
  for (int64_t t0 = (int64_t)blockIdx.x * TPB; t0 < a.T; t0 += stride) {
    const int64_t t = t0 + g, row = t * a.E;
    const RowRaw<VEC, NCH> raw = next;
    const bool live = mask != 0;
    if (t0 + stride < a.T) load(t + stride);
    Cols<VEC> p[NCH];
    row_softmax<VEC, LPT, NCH>(raw, a.f32, a.E, l, live, p);
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
// lanes as hold the row, others and the shortest one logit at a time.
template <class F>
hipError_t by_experts(int E, F&& f) {
  using std::integral_constant;
#define LX_E(V, L, N) f(integral_constant<int, V>{}, integral_constant<int, L>{}, integral_constant<int, N>{})
  if (E <= 8) return LX_E(1, 8, 1);
  if (E <= 16) return LX_E(1, 16, 1);
  if (E <= 32) return LX_E(1, 32, 1);
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

int lanes_per_token(int E) {
  int n = 0;
  (void)by_experts(E, [&](auto, auto lpt, auto) {
    n = decltype(lpt)::value;
    return hipSuccess;
  });
  return n;
}

}  // namespace

// A round is the tokens that a workgroup takes at once. One workgroup up to
// three rounds, which take about as long as the second launch that it saves;
// from there on as many as have two rounds each, at most 128, which is what one
// workgroup joins in a few microseconds.
int balance_blocks(int T, int E) {
  const int64_t tpb = kFwd / lanes_per_token(E), rounds = (T + tpb - 1) / tpb;
  return rounds <= 3 ? 1 : (int)std::min<int64_t>((rounds + 1) / 2, 128);
}

hipError_t launch_balance(const BalanceArgs& a, hipStream_t s) {
  return by_experts(a.E, [&](auto v, auto l, auto n) {
    k_balance<decltype(v)::value, decltype(l)::value, decltype(n)::value><<<a.blocks, kFwd, 0, s>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_balance_sum(const BalanceArgs& a, hipStream_t s) {
  k_balance_sum<<<1, kFwd, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_balance_grad(const BalanceArgs& a, hipStream_t s) {
  const int tpb = kThreads / lanes_per_token(a.E);
  const int grid = (int)std::min<int64_t>(((int64_t)a.T + tpb - 1) / tpb, 1024);
  return by_experts(a.E, [&](auto v, auto l, auto n) {
    k_balance_grad<decltype(v)::value, decltype(l)::value, decltype(n)::value><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace lx
