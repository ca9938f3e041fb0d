// A layer of experts in 4 bits for a few tokens, in two launches (formulas in
// lorex_block.h). Bound by reading the chosen experts' weights once.
//
// The activations are not rounded: the weights are read back to bf16, which holds
// them exactly, and multiplied on the bf16 matrix instructions with bf16 terms that
// add up to the activation (one for bf16, two or three for fp32: 8 bits each).
//
// A wavefront has 16 weight rows and the tokens that chose their expert as columns,
// 16 at a time; lane l holds row (token) l % 16 and, of the 128 values of a step,
// block l / 16: 16 bytes of codes under one scale, which are four instructions'
// operands. The sum over K does not mind that an instruction's 32 values are
// then 8 of each block.
#include "lx_block.h"
#include "lx_mx8.h"
#include "lx_vec.h"

#include <algorithm>
#include <type_traits>

namespace lx {
namespace {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef uint32_t vu4w __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t vu2 __attribute__((ext_vector_type(2)));

// 8 codes under the scale f, as bf16.
__device__ __forceinline__ bf8 read8(uint32_t codes, float f) {
  const vb2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 1),
            c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 3);
  return bf8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// An fp32 value as three bf16 terms that add up to it exactly: its upper 8 bits (cut
// off, so that none overflows), those of the rest (rounded to nearest: without the
// third term the error is at most 2^-16 of the value), and the remainder. Infinities
// and NaN are the first term alone.
struct Terms {
  uint32_t t[3];  // in the upper halves
};
__device__ __forceinline__ Terms terms(float x) {
  Terms r;
  const uint32_t b = __float_as_uint(x);
  r.t[0] = b & 0xFFFF0000u;
  const float x1 = x - __uint_as_float(r.t[0]);
  r.t[1] = pack_bf16(0.f, x1);
  r.t[2] = __float_as_uint(x1 - __uint_as_float(r.t[1]));
  if ((b & 0x7F800000u) == 0x7F800000u) {
    r.t[0] |= b & 0x7FFFFFu ? 0x7FC00000u : 0u;
    r.t[1] = r.t[2] = 0;
  }
  return r;
}
__device__ __forceinline__ uint32_t two(uint32_t lo, uint32_t hi) { return lo >> 16 | (hi & 0xFFFF0000u); }

// 8 activations from column c of a row (null: zeros) as N terms.
template <int N, bool F32>
struct Acts {
  vu4 t[N];
  __device__ __forceinline__ void load(const void* row, int c, int K) {
#pragma unroll
    for (int n = 0; n < N; ++n) t[n] = vu4{0, 0, 0, 0};
    if (!row || c >= K) return;
    if constexpr (F32) {
      static_assert(N == 3, "");
      const vu4* const p = (const vu4*)((const float*)row + c);
      const vu4 a = p[0], b = p[1];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Terms u = terms(__uint_as_float(j < 2 ? a[2 * j] : b[2 * j - 4])), v = terms(__uint_as_float(j < 2 ? a[2 * j + 1] : b[2 * j - 3]));
#pragma unroll
        for (int n = 0; n < 3; ++n) t[n][j] = two(u.t[n], v.t[n]);
      }
    } else {
      t[0] = *(const vu4*)((const uint16_t*)row + c);
    }
  }
};

__device__ __forceinline__ vf4 mfma(bf8 w, const vu4& a, vf4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf8, a), acc, 0, 0, 0);
}

// Which tokens chose expert e: lane t looks at token t's k ids. The token's weight is
// the sum over its slots of e (the same expert twice counts twice), its row of the
// hidden activations the first of them.
struct Chosen {
  uint64_t mask;  // uniform: tokens with a slot of e
  float weight;   // this lane's token
  int row;
};
__device__ __forceinline__ Chosen chosen(const FewArgs& a, int e) {
  const int t = threadIdx.x & 63;
  Chosen c{0, 0.f, -1};
  if (t < a.T)
    for (int j = a.k - 1; j >= 0; --j)
      if (a.ids[t * a.k + j] == e) {
        c.weight += a.weights[t * a.k + j];
        c.row = t * a.k + j;
      }
  c.mask = __ballot(c.row >= 0);
  return c;
}

// Expert u of those that may have tokens, -1 if there is none: every expert in turn
// where there are no more of them than slots, else the slots, each expert at the
// first of its own.
__device__ __forceinline__ int expert_of(const FewArgs& a, int u, Chosen& c) {
  const bool by_slot = a.units != a.E;
  const int e = __builtin_amdgcn_readfirstlane(by_slot ? a.ids[u] : u);
  if (e < 0 || e >= a.E) return -1;
  c = chosen(a, e);
  if (!c.mask) return -1;
  if (by_slot && __builtin_amdgcn_readlane(c.row, __builtin_ctzll(c.mask)) != u) return -1;
  return e;
}

// Gate and up projections, SwiGLU and the router's weight: 16 hidden columns of one
// expert per workgroup, whose four wavefronts share K and add their sums in order.
// The results go to a.hidden as three bf16 terms, row (token, first slot) by row.
template <bool F32>
__global__ __launch_bounds__(256) void k_few_up(const FewArgs a) {
  constexpr int N = F32 ? 3 : 1;
  __shared__ float part[3][2][256];
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles = (a.f + 15) / 16, u = blockIdx.x / tiles, n0 = blockIdx.x % tiles * 16;
  Chosen c{};
  const int e = expert_of(a, u, c);
  if (n0 == 0 && wave == 0) {  // for the second launch
    if (lane == 0) a.unit_mask[u] = e < 0 ? 0 : c.mask, a.unit_expert[u] = e;
    if (e >= 0 && c.row >= 0) a.unit_row[u * 64 + lane] = c.row;
  }
  if (e < 0) return;
  const int dp = LX_MX4_KP(a.d), cp = dp / 2, sp = dp / 32, steps = dp / 128;
  const int rank = __popcll(c.mask & ((1ull << lane) - 1));
  // the tokens in order, the chosen ones first: lane i learns the i-th
  const int count = __popcll(c.mask);
  const int token = __builtin_amdgcn_ds_permute((c.row >= 0 ? rank : count + lane - rank) * 4, lane);
  const int64_t grow = (int64_t)e * 2 * a.f + min(n0 + l16, a.f - 1);
  const uint8_t* const G = a.gu + grow * cp + q * 16;
  const uint8_t* const Gs = a.gu_s + grow * sp + q;
  const int64_t up = (int64_t)a.f * cp, ups = (int64_t)a.f * sp;
  const int k0 = steps * wave / 4, k1 = steps * (wave + 1) / 4;
  for (int c0 = 0; c0 < count; c0 += 16) {
    const int col = c0 + l16;
    const int t = __builtin_amdgcn_ds_bpermute(min(col, count - 1) * 4, token);
    const void* const x = col < count ? (const uint8_t*)a.x + (int64_t)t * a.d * (F32 ? 4 : 2) : nullptr;
    vf4 ag = {0.f, 0.f, 0.f, 0.f}, au = ag;
    auto batch = [&](auto cnt, int k) __attribute__((always_inline)) {
      constexpr int U = decltype(cnt)::value;
      vu4 wg[U], wu[U];
      uint32_t sg[U], su[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        wg[i] = *(const vu4*)(G + (int64_t)(k + i) * 64);
        wu[i] = *(const vu4*)(G + up + (int64_t)(k + i) * 64);
        sg[i] = Gs[(k + i) * 4];
        su[i] = Gs[ups + (k + i) * 4];
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const float fg = mx_scale(sg[i]), fu = mx_scale(su[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          Acts<N, F32> v;
          v.load(x, (k + i) * 128 + q * 32 + j * 8, a.d);
          const bf8 g = read8(wg[i][j], fg), w = read8(wu[i][j], fu);
#pragma unroll
          for (int n = N - 1; n >= 0; --n) {
            ag = mfma(g, v.t[n], ag);
            au = mfma(w, v.t[n], au);
          }
        }
      }
    };
    int k = k0;
    for (; k + 4 <= k1; k += 4) batch(std::integral_constant<int, 4>{}, k);
    for (; k < k1; ++k) batch(std::integral_constant<int, 1>{}, k);
    if (wave > 0) {
      *(vf4*)&part[wave - 1][0][lane * 4] = ag;
      *(vf4*)&part[wave - 1][1][lane * 4] = au;
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int w = 0; w < 3; ++w) {
        ag += *(const vf4*)&part[w][0][lane * 4];
        au += *(const vf4*)&part[w][1][lane * 4];
      }
      const float weight = __uint_as_float(__builtin_amdgcn_ds_bpermute(t * 4, __float_as_uint(c.weight)));
      const int row = __builtin_amdgcn_ds_bpermute(t * 4, c.row);
      const int n = n0 + q * 4;  // (f is a multiple of 8: all four columns exist or none)
      Terms h[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) h[j] = terms(silu(ag[j]) * au[j] * weight);
      if (col < count && n < a.f) {
        uint16_t* const p = a.hidden + (int64_t)row * 3 * a.f + n;
#pragma unroll
        for (int m = 0; m < 3; ++m)
          *(vu2*)(p + m * a.f) = vu2{two(h[0].t[m], h[1].t[m]), two(h[2].t[m], h[3].t[m])};
      }
    }
    __syncthreads();
  }
}

// Down projections and the sum over a token's experts: 16 columns of the output per
// workgroup, for all tokens. The NW wavefronts share the steps of all chosen
// experts, a contiguous part each, with sums of their own in LDS for every token,
// which are added in order at the end. TERMS of the hidden activations are
// multiplied: for a bf16 output two (2^-16 of a value at most, next to the 2^-9 that
// the output is rounded by), for fp32 all three.
constexpr int kDownWaves = 16;
template <int TERMS>
__global__ __launch_bounds__(kDownWaves * 64) void k_few_down(const FewArgs a) {
  extern __shared__ float sums[];  // [kDownWaves][T][16]
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * 16;
  float* const mine = sums + wave * a.T * 16;
  for (int i = lane; i < a.T * 16; i += 64) mine[i] = 0.f;
  const int fp = LX_MX4_KP(a.f), cp = fp / 2, sp = fp / 32, steps = fp / 128;
  int live = 0;
  for (int u0 = 0; u0 < a.units; u0 += 64) live += __popcll(__ballot(u0 + lane < a.units && a.unit_mask[min(u0 + lane, a.units - 1)] != 0));
  const int all = live * steps;
  int at = (int)((int64_t)all * wave / kDownWaves);
  const int end = (int)((int64_t)all * (wave + 1) / kDownWaves);
  int before = 0;  // live units before u0
  for (int u0 = 0; u0 < a.units && at < end; u0 += 64) {
    const uint64_t m = u0 + lane < a.units ? a.unit_mask[u0 + lane] : 0;
    uint64_t left = __ballot(m != 0);
    const int here = __popcll(left);
    for (int i = before; left && at < end; ++i, left &= left - 1) {
      if (at >= (i + 1) * steps) continue;
      const int src = __builtin_ctzll(left), u = u0 + src;
      const uint64_t mask = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(m >> 32), src) << 32 |
                            (uint32_t)__builtin_amdgcn_readlane((int)m, src);
      const int e = __builtin_amdgcn_readfirstlane(a.unit_expert[u]);
      const int k0 = at - i * steps, k1 = min(end - i * steps, steps);
      at = i * steps + k1;
      const int count = __popcll(mask), rank = __popcll(mask & ((1ull << lane) - 1));
      const bool has = mask >> lane & 1;
      const int token = __builtin_amdgcn_ds_permute((has ? rank : count + lane - rank) * 4, lane);
      const int64_t brow = (int64_t)e * a.d + min(n0 + l16, a.d - 1);
      const uint8_t* const D = a.down + brow * cp + q * 16;
      const uint8_t* const Ds = a.down_s + brow * sp + q;
      for (int c0 = 0; c0 < count; c0 += 16) {
        const int col = c0 + l16;
        const int t = __builtin_amdgcn_ds_bpermute(min(col, count - 1) * 4, token);
        const int row = col < count ? a.unit_row[u * 64 + t] : -1;
        const uint16_t* const h = row >= 0 ? a.hidden + (int64_t)row * 3 * a.f : nullptr;
        vf4 acc = {0.f, 0.f, 0.f, 0.f};
        auto batch = [&](auto cnt, int k) __attribute__((always_inline)) {
          constexpr int U = decltype(cnt)::value;
          vu4 w[U];
          uint32_t s[U];
#pragma unroll
          for (int i = 0; i < U; ++i) {
            w[i] = *(const vu4*)(D + (int64_t)(k + i) * 64);
            s[i] = Ds[(k + i) * 4];
          }
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const float f = mx_scale(s[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const bf8 v = read8(w[i][j], f);
#pragma unroll
              for (int n = TERMS - 1; n >= 0; --n) {
                Acts<1, false> x;
                x.load(h ? h + n * a.f : nullptr, (k + i) * 128 + q * 32 + j * 8, a.f);
                acc = mfma(v, x.t[0], acc);
              }
            }
          }
        };
        int k = k0;
        for (; k + 4 <= k1; k += 4) batch(std::integral_constant<int, 4>{}, k);
        for (; k < k1; ++k) batch(std::integral_constant<int, 1>{}, k);
        if (col < count) *(vf4*)(mine + t * 16 + q * 4) += acc;
      }
    }
    before += here;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.T * 16; i += kDownWaves * 64) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kDownWaves; ++w) s += sums[w * a.T * 16 + i];
    const int n = n0 + (i & 15);
    if (n < a.d) {
      const int64_t o = (int64_t)(i >> 4) * a.d + n;
      if (a.out_f32)
        ((float*)a.out)[o] = s;
      else
        ((uint16_t*)a.out)[o] = (uint16_t)pack_bf16(s, 0.f);
    }
  }
}

}  // namespace

hipError_t launch_few_up(const FewArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)a.units * ((a.f + 15) / 16);
  if (a.x_f32)
    k_few_up<true><<<grid, 256, 0, s>>>(a);
  else
    k_few_up<false><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_few_down(const FewArgs& a, hipStream_t s) {
  const unsigned grid = (a.d + 15) / 16, lds = kDownWaves * a.T * 16 * sizeof(float);
  if (a.out_f32)
    k_few_down<3><<<grid, kDownWaves * 64, lds, s>>>(a);
  else
    k_few_down<2><<<grid, kDownWaves * 64, lds, s>>>(a);
  return hipGetLastError();
}

}  // namespace lx
