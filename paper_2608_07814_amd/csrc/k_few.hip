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
// then 8 of each block. Loaded by these lanes, each quarter of a wavefront would touch
// 16 rows for 16 bytes each (what the first-level cache looks up took two thirds of its
// cycles, at 2.9 TB/s); so the codes go to LDS in whole lines first, to a place that is
// the wavefront's own, and the scales, 16 bytes a row, to 16 lanes.
#include "lx_block.h"
#include "lx_device_once.h"
#include "lx_groups.h"
#include "lx_mx8.h"
#include "lx_silu.h"
#include "lx_vec.h"

#include <algorithm>
#include <type_traits>

namespace lx {
namespace {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef uint32_t vu4w __attribute__((ext_vector_type(4), aligned(4)));

// 8 codes under the scale f, as bf16.
__device__ __forceinline__ bf8 read8(uint32_t codes, float f) {
  const vb2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 1),
            c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 3);
  return bf8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// An fp32 value as three bf16 terms that add up to it exactly: its upper 8 bits (cut
// off, so that none overflows), those of the rest (rounded to nearest), and the
// remainder. Infinities and NaN are the first term alone.
constexpr int kTerms = 3;
struct Terms {
  uint32_t t[kTerms];  // in the upper halves
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

// 8 activations: as they are loaded, from column c of the row that begins at byte `row` of
// x (T d is at most 2^26; not `there`: zeros), and as terms.
template <bool F32>
struct Acts {
  static constexpr int N = F32 ? kTerms : 1, R = F32 ? 2 : 1;
  vu4 r[R];
  __device__ __forceinline__ void load(const void* x, uint32_t row, bool there, int c, int K) {
#pragma unroll
    for (int i = 0; i < R; ++i) r[i] = vu4{0, 0, 0, 0};
    if (!there || c >= K) return;
    const vu4* const p = (const vu4*)((const uint8_t*)x + (row + (uint32_t)c * (F32 ? 4 : 2)));
#pragma unroll
    for (int i = 0; i < R; ++i) r[i] = p[i];
  }
  // terms() of 8 values, whose infinities and NaN, if there are any, are put right
  // afterwards: they leave a NaN in the sum of the rests
  __device__ __forceinline__ void split(vu4 (&t)[N]) const {
    if constexpr (!F32) {
      t[0] = r[0];
    } else {
      float all = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t u = r[j / 2][j % 2 * 2], v = r[j / 2][j % 2 * 2 + 1];
        const float ru = __uint_as_float(u) - __uint_as_float(u & 0xFFFF0000u), rv = __uint_as_float(v) - __uint_as_float(v & 0xFFFF0000u);
        all += ru + rv;
        t[0][j] = two(u, v);
        t[1][j] = pack_bf16(ru, rv);
        t[2][j] = two(__float_as_uint(ru - __uint_as_float(t[1][j] << 16)), __float_as_uint(rv - __uint_as_float(t[1][j] & 0xFFFF0000u)));
      }
      if (!(all == all)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const Terms u = terms(__uint_as_float(r[j / 2][j % 2 * 2])), v = terms(__uint_as_float(r[j / 2][j % 2 * 2 + 1]));
#pragma unroll
          for (int n = 0; n < kTerms; ++n) t[n][j] = two(u.t[n], v.t[n]);
        }
      }
    }
  }
};

// Lane l of each 16 gets what lane l + R of them has.
template <int R>
__device__ __forceinline__ vu4 from_right(const vu4& x) {
  if constexpr (R == 0) return x;
  vu4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x[i], 0x120 + (16 - R) % 16, 0xF, 0xF, false);
  return r;
}

__device__ __forceinline__ vf4 mfma(bf8 w, const vu4& a, vf4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf8, a), acc, 0, 0, 0);
}

// kBatch steps of 16 rows of weights, on their way through LDS. `steps`: of a row.
constexpr int kBatch = 4, kStage = 16 * kBatch * 64;

// Asks for the codes of steps k .. k + n - 1 (n of 1 .. kBatch) of rows row .. row + 15 (of
// rows up to `last`; later ones repeat it) into `stage`: two steps are a line of 128
// bytes of a row, whose 16-byte chunks are XORed with (row / 2) % 8, so that the 16
// lanes that a read serves together hit different banks. Of a single step the upper
// chunks repeat the lower ones.
__device__ __forceinline__ void ask_codes(const uint8_t* codes, int64_t row, int last, int steps, int k, int n, const uint8_t* stage) {
  const int lane = threadIdx.x & 63;
  const uint8_t* const base = codes + row * ((int64_t)steps * 64) + (int64_t)k * 64;
#pragma unroll
  for (int p = 0; p < kBatch / 2; ++p)
    if (2 * p < n) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = 8 * j + lane / 8, c = (lane ^ (r >> 1)) & 7;
        const uint32_t at = (uint32_t)min(r, last) * (uint32_t)(steps * 64) + (2 * p + 1 < n ? c : c & 3) * 16;
        load_lds<16>(base + p * 128, at, stage + p * 2048 + j * 1024);
      }
    }
}
// This lane's codes of step i of the batch.
__device__ __forceinline__ vu4 codes_of(const uint8_t* stage, int i) {
  const int l16 = threadIdx.x & 15, q = (threadIdx.x & 63) >> 4;
  return *(const vu4*)(stage + (i >> 1) * 2048 + l16 * 128 + ((((i & 1) * 4 + q) ^ (l16 >> 1)) & 7) * 16);
}

// The scales of steps k .. k + n - 1: lanes 0 .. 15 of `lanes` load a row's (4 bytes a
// step) and hand them on. A row's last 16 bytes are loaded where fewer are left.
struct Scales {
  vu4 w;
};
__device__ __forceinline__ Scales ask_scales(const uint8_t* row, int steps, int k, int n, bool lanes) {
  Scales s{};
  if (lanes) {
    if (steps >= 4) {
      s.w = *(const vu4w*)(row + min(k, steps - 4) * 4);
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < n) s.w[i] = *(const uint32_t*)(row + (k + i) * 4);
    }
  }
  return s;
}
// What this lane's block of step i stands under; `from`: the lane that has its row.
__device__ __forceinline__ float scale_of(const Scales& s, int steps, int k, int i, int from) {
  const int late = steps >= 4 ? max(k - (steps - 4), 0) : 0, q = (threadIdx.x & 63) >> 4;
  uint32_t w = s.w[0];
#pragma unroll
  for (int j = 1; j < 4; ++j) w = i + late == j ? s.w[j] : w;
  return mx_scale((uint32_t)__builtin_amdgcn_ds_bpermute(from * 4, (int)w) >> (8 * q) & 255);
}
__device__ __forceinline__ void all_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void all_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Which tokens chose expert e: lane t looks at token t's k ids. Its hidden activations
// are a row of their own: the tokens of an expert follow each other from `base` on, the
// number of slots of lower experts.
struct Chosen {
  uint64_t mask;  // uniform: tokens with a slot of e
  int base;       // uniform
  int slot;       // this lane's token's first slot of e, -1: none
};
// f(slot, id) for the slots of lane t's token, in order.
template <class F>
__device__ __forceinline__ void for_slots(const FewArgs& a, F&& f) {
  const int t = threadIdx.x & 63;
  if (t >= a.T) return;
  int j = t * a.k;
  const int end = j + a.k;
  for (; j + 4 <= end; j += 4) {
    const vu4w id = *(const vu4w*)(a.ids + j);
#pragma unroll
    for (int i = 0; i < 4; ++i) f(j + i, (int)id[i]);
  }
  for (; j < end; ++j) f(j, a.ids[j]);
}
__device__ __forceinline__ Chosen chosen(const FewArgs& a, int e) {
  Chosen c{0, 0, -1};
  int less = 0;
  for_slots(a, [&](int slot, int id) __attribute__((always_inline)) {
    if (id == e && c.slot < 0) c.slot = slot;
    less += id >= 0 && id < e;
  });
  c.mask = __ballot(c.slot >= 0);
  c.base = __builtin_amdgcn_readfirstlane((int)lane_sum<64>((float)less));  // (at most 2048)
  return c;
}

// The tokens of a mask in order: lane i learns the i-th (the others follow).
__device__ __forceinline__ int token_list(uint64_t mask) {
  const int lane = threadIdx.x & 63, rank = __popcll(mask & ((1ull << lane) - 1));
  return __builtin_amdgcn_ds_permute((mask >> lane & 1 ? rank : __popcll(mask) + lane - rank) * 4, lane);
}

// Where the hidden activations lie: those of up to 16 tokens of an expert (its tokens
// from c0 on) together, term by term, step by step of 128, and within a step so that what
// a load instruction of the second launch takes, 8 values of each block of every token,
// is contiguous. `cols`: the tokens of the 16.
__device__ __forceinline__ uint16_t* hidden_of(const FewArgs& a, int base, int c0) {
  return a.hidden + (int64_t)(base + c0) * kTerms * LX_MX4_KP(a.f);
}
__device__ __forceinline__ int64_t hidden_at(int fp, int term, int step, int j, int q, int cols, int col) {
  return ((int64_t)term * fp / 8 + ((step * 4 + j) * 4 + q)) * cols * 8 + col * 8;
}

// Gate and up projections, SwiGLU and the router's weight: 16 hidden columns of one
// expert per workgroup, whose four wavefronts share K and meet in LDS. A unit is an
// expert where there are no more of them than slots, else a slot, of which each expert's
// first does the work. Many short workgroups hide each other's waits: several tiles to
// a workgroup in turn, the next one's weights on their way, took a third longer. The
// results go to a.hidden as bf16 terms. Experts of 14336 x 4096, 5 tokens on 6 or 7 of
// them: 90 to 96 us, the weights at 4.3 TB/s; of 768 x 2048, 61 tokens on 90 of 128: 47 us, 3.2
// (the first-level cache is asked for something in every cycle: by 16 loads of activations
// a batch, most of whose lanes have no token, next to 8 of codes). Both launches with fp32
// activations take 20 to 35% longer, for the instructions that split them. Tried and no
// faster: a tile of its own for each wavefront where rows are short; x through LDS (64
// tokens on 8 experts 182 for 205, most others a little slower); four sets of 16 tokens
// on the same codes (both launches, with two terms of the hidden activations: 64 tokens on 8
// experts 338 for 349, 61 on 128 89 for 85).
template <bool F32>
__global__ __launch_bounds__(256, 4) void k_few_up(const FewArgs a) {
  constexpr int N = F32 ? kTerms : 1;
  __shared__ __attribute__((aligned(16))) uint8_t stage[4][2][kStage];
  __shared__ float weight[64];
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fp = LX_MX4_KP(a.f), u = blockIdx.y, n0 = blockIdx.x * 16;
  // (the second launch counts the workgroups that are done with a column tile)
  if (n0 == 0 && u == 0)
    for (int i = threadIdx.x; i < a.counters; i += 256) a.counter[i] = 0;
  const bool by_slot = a.units != a.E;
  const int e = __builtin_amdgcn_readfirstlane(by_slot ? a.ids[u] : u);
  const bool valid = e >= 0 && e < a.E;
  Chosen c{0, 0, -1};
  if (valid) c = chosen(a, e);
  const bool live = c.mask && !(by_slot && __builtin_amdgcn_readlane(c.slot, __builtin_ctzll(c.mask | 1ull << 63)) != u);
  if (n0 == 0 && threadIdx.x == 0)  // for the second launch
    a.unit[u] = FewUnit{live ? e : -1, c.base, c.mask};
  if (!live) return;
  const int count = __popcll(c.mask), token = token_list(c.mask);
  // a token's weight is the sum over its slots of e (the same expert twice counts twice)
  if (wave == 0) {
    float s = 0.f;
    for_slots(a, [&](int slot, int id) __attribute__((always_inline)) {
      const float w = a.weights[slot];
      s += id == e ? w : 0.f;
    });
    if (c.slot >= 0) weight[__popcll(c.mask & ((1ull << lane) - 1))] = s;
  }
  // (past f the rows are padded with zeros)
  const bool padding = n0 >= a.f;
  const int steps = LX_MX4_KP(a.d) / 128, sp = steps * 4, k0 = steps * wave / 4, k1 = steps * (wave + 1) / 4;
  const int64_t row = (int64_t)e * 2 * a.f + (padding ? 0 : n0);
  const int last = padding ? 0 : min(a.f - 1 - n0, 15);
  // lanes 0 .. 15: scales of the gate rows, 16 .. 31: of the up rows
  const uint8_t* const my_scales = a.gu_s + (row + (lane & 16 ? a.f : 0) + min(l16, last)) * sp;
  uint8_t *const sg = stage[wave][0], *const su = stage[wave][1];
  for (int c0 = 0; c0 < count; c0 += 16) {
    const int cols = min(count - c0, 16);
    vf4 ag = {0.f, 0.f, 0.f, 0.f}, au = ag;
    for (int k = k0; k < k1 && !padding; k += kBatch) {
      const int n = min(k1 - k, kBatch);
      all_read();  // (the batch before)
      ask_codes(a.gu, row, last, steps, k, n, sg);
      ask_codes(a.gu, row + a.f, last, steps, k, n, su);
      const Scales sc = ask_scales(my_scales, steps, k, n, lane < 32);
      // At most G tokens: the lanes of the columns that they leave load, and split into
      // terms, what the following 16 / G - 1 instructions take. (fp32: 5 tokens on experts
      // of 14336 x 4096 181 us for 212, both launches; in bf16, with nothing to split, 100 for
      // 97 in this one.)
      auto products = [&](auto most) __attribute__((always_inline)) {
        constexpr int G = decltype(most)::value, PER = 16 / G, L = 4 / PER;
        int l16 = lane & 15;
        if (F32) asm volatile("" : "+v"(l16));  // (what follows from it is not kept over the batches)
        const int t = __builtin_amdgcn_ds_bpermute(min(c0 + l16 % G, count - 1) * 4, token);
        const uint32_t x = (uint32_t)t * (uint32_t)a.d * (F32 ? 4 : 2);
        const bool there = l16 % G < cols;
        // activations: of all steps (bf16), or two loads at a time, the next two on their
        // way (fp32)
        constexpr int C = F32 ? 2 : 4 * L, CHUNKS = 4 * L / C;
        Acts<F32> v[F32 ? 2 : 1][C];
        auto ask = [&](int c) __attribute__((always_inline)) {
#pragma unroll
          for (int s = 0; s < C; ++s) {
            const int i = (c * C + s) / L, l = (c * C + s) % L;
            if (i < n) v[c % 2][s].load(a.x, x, there, (k + i) * 128 + q * 32 + (l * PER + l16 / G) * 8, a.d);
          }
        };
        ask(0);
        all_landed();
        float fg = 0.f, fu = 0.f;
        vu4 wg = {0, 0, 0, 0}, wu = wg;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          if (c + 1 < CHUNKS) ask(c + 1);
#pragma unroll
          for (int s = 0; s < C; ++s) {
            const int i = (c * C + s) / L, l = (c * C + s) % L;
            if (i < n) {
              if (l == 0) {
                fg = scale_of(sc, steps, k, i, l16);
                fu = scale_of(sc, steps, k, i, 16 + l16);
                wg = codes_of(sg, i);
                wu = codes_of(su, i);
              }
              vu4 t[N];
              v[c % 2][s].split(t);
              auto one = [&](auto jj) __attribute__((always_inline)) {
                constexpr int J = decltype(jj)::value;
                if constexpr (J < PER) {
                  const bf8 g = read8(wg[l * PER + J], fg), z = read8(wu[l * PER + J], fu);
#pragma unroll
                  for (int m = N - 1; m >= 0; --m) {
                    const vu4 u = from_right<J * G>(t[m]);
                    ag = mfma(g, u, ag);
                    au = mfma(z, u, au);
                  }
                }
              };
              one(std::integral_constant<int, 0>{});
              one(std::integral_constant<int, 1>{});
              one(std::integral_constant<int, 2>{});
              one(std::integral_constant<int, 3>{});
            }
          }
        }
      };
      if (F32 && cols <= 4)
        products(std::integral_constant<int, 4>{});
      else if (F32 && cols <= 8)
        products(std::integral_constant<int, 8>{});
      else
        products(std::integral_constant<int, 16>{});
    }
    all_read();
    // (the sums meet where the codes were)
    float* const part = (float*)sg;
    *(vf4*)(part + l16 * 16 + q * 4) = ag;
    *(vf4*)(part + 256 + l16 * 16 + q * 4) = au;
    __syncthreads();
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // (what follows from it is not kept over the products)
    const int e8 = tid & 7, col = tid / 8 % 16, n = tid / 128 * 8 + e8;
    if (col < cols) {
      float g = 0.f, z = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* const p = (const float*)stage[i][0] + col * 16 + n;
        g += p[0];
        z += p[256];
      }
      const int at = n0 + n;
      const Terms h = terms(at < a.f ? silu(g) * z * weight[c0 + col] : 0.f);
      uint16_t* const p = hidden_of(a, c.base, c0) + e8;
#pragma unroll
      for (int m = 0; m < kTerms; ++m) p[hidden_at(fp, m, at / 128, at / 8 % 4, at / 32 % 4, cols, col)] = (uint16_t)(h.t[m] >> 16);
    }
    __syncthreads();
  }
}

// Device-scope coherent store and load: another XCD's workgroup that reads the place
// after this access has completed sees its value.
__device__ __forceinline__ void store_dev(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float load_dev(const float* p) {
  return __hip_atomic_load(const_cast<float*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Down projections and the sum over a token's experts: 16 columns of the output, for
// all tokens, by a.splits workgroups. Their wavefronts share the steps of all chosen
// experts, batch by batch in turn, with sums of their own in LDS for every token, which
// are added in order at the end: first over a workgroup's wavefronts, then, by
// the workgroup that is done last, over the workgroups. What workgroups hand each other is
// stored and loaded coherently and complete before the counter is raised, which is all
// the order that it needs (fences, which write back and empty whole caches, took the
// launch from 93 to 205 us).
// All terms of the hidden activations are multiplied, for a bf16 output too (with two,
// 2^-16 of a value at most, too little is left where sums cancel). They are
// columns of one instruction side by side, PACKED tokens at a time, so that a batch's
// activations fit in registers and are asked for together with its codes: there is one
// wait to a batch. 5 tokens on 6 or 7 experts of 14336 x 4096 65 us, the weights at 3.1
// TB/s; 61 tokens on 90 experts of 768 x 2048 51, 1.5 TB/s (with two terms, eight tokens to an
// instruction, 36); one token on 8 of these 8. Term by term, a step ahead, all with two:
// 87 for 66, 42 for 36. A workgroup to an expert and 16 to 64 columns,
// its products joined by the last one or by a third launch, took 30% or 0 to 20% longer.
constexpr int kDownWaves = 16;
__global__ __launch_bounds__(kDownWaves * 64, 4) void k_few_down(const FewArgs a) {
  constexpr int U = kBatch, PACKED = 16 / kTerms;
  __shared__ __attribute__((aligned(16))) uint8_t stage[kDownWaves][kStage];
  // [kDownWaves][T][16] sums, then three words for each unit with tokens
  extern __shared__ __attribute__((aligned(16))) float sums[];
  int* const list = (int*)(sums + kDownWaves * a.T * 16);
  __shared__ int done;
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % a.splits, n0 = blockIdx.x / a.splits * 16;
  float* const mine = sums + wave * a.T * 16;
  for (int i = lane; i < a.T * 16; i += 64) mine[i] = 0.f;
  // every wavefront counts all units, each writes some
  int live = 0;
#pragma unroll 2
  for (int u0 = 0; u0 < a.units; u0 += 64) {
    const FewUnit m = u0 + lane < a.units ? a.unit[u0 + lane] : FewUnit{-1, 0, 0};
    const uint64_t there = __ballot(m.expert >= 0);
    if (m.expert >= 0 && (u0 >> 6) % kDownWaves == wave) {
      int* const at = list + 3 * (live + __popcll(there & ((1ull << lane) - 1)));
      at[0] = m.expert | m.base << 16;  // (E is at most 8192, a row below 2048)
      at[1] = (int)m.mask;
      at[2] = (int)(m.mask >> 32);
    }
    live += __popcll(there);
  }
  __syncthreads();
  const int fp = LX_MX4_KP(a.f), steps = fp / 128, sp = steps * 4;
  // Batch b is steps kBatch (b % batches) .. of live unit b / batches: wavefronts that run
  // together read neighbouring parts of the same rows.
  const int batches = (steps + U - 1) / U, all = live * batches;
  const int last = min(a.d - 1 - n0, 15);
  int token = 0, count = 0, base = 0, expert = 0, unit = -1;
  vf4 acc = {0.f, 0.f, 0.f, 0.f};
  // acc into the sums of tokens c0 .. to - 1
  auto flush = [&](int c0, int to) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {  // the terms' sums, the least first
      float s = 0.f;
#pragma unroll
      for (int m = kTerms - 1; m > 0; --m) s += __uint_as_float(__builtin_amdgcn_ds_bpermute((lane + m * PACKED) * 4, (int)__float_as_uint(acc[r])));
      acc[r] += s;
    }
    const int t = __builtin_amdgcn_ds_bpermute(min(c0 + l16, count - 1) * 4, token);
    if (c0 + l16 < to) *(vf4*)(mine + t * 16 + q * 4) += acc;
    acc = vf4{0.f, 0.f, 0.f, 0.f};
  };
  for (int b = split * kDownWaves + wave; b < all; b += a.splits * kDownWaves) {
    const int i = b / batches, k = (b - i * batches) * U, n = min(steps - k, U);
    if (i != unit) {
      if (unit >= 0 && count <= PACKED) flush(0, count);
      unit = i;
      const int m = __builtin_amdgcn_readfirstlane(list[3 * i]);
      expert = m & 0xFFFF;
      base = m >> 16;
      const uint64_t mask = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane(list[3 * i + 2]) << 32 |
                            (uint32_t)__builtin_amdgcn_readfirstlane(list[3 * i + 1]);
      count = __popcll(mask);
      token = token_list(mask);
    }
    const int64_t row = (int64_t)expert * a.d + n0;
    all_read();  // (the batch before)
    ask_codes(a.down, row, last, steps, k, n, stage[wave]);
    const Scales sc = ask_scales(a.down_s + (row + min(l16, last)) * sp, steps, k, n, lane < 16);
    for (int c0 = 0, to; c0 < count; c0 = to) {
      const int g = c0 & ~15, cols = min(count - g, 16);
      to = min(min(c0 + PACKED, g + 16), count);
      const uint8_t* const h = (const uint8_t*)hidden_of(a, base, g) + hidden_at(fp, 0, k, 0, 0, cols, c0 - g) * 2;
      int l = lane;
      asm volatile("" : "+v"(l));  // (what follows from it is not kept over the batches)
      // (columns without a token, and steps past the last, repeat some that are there)
      const int m = min((l & 15) / PACKED, kTerms - 1), col = min((l & 15) % PACKED, to - c0 - 1);
      const uint32_t own = ((uint32_t)(m * (fp / 8) + (l >> 4)) * cols + col) * 16;
      vu4 x[U][4];
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = *(const vu4*)(h + (own + (uint32_t)((min(i, n - 1) * 4 + j) * 64 * cols)));
      all_landed();  // (for the first tokens; it also keeps the codes from being read ahead of the loop)
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (i < n) {
          const float f = scale_of(sc, steps, k, i, l16);
          const vu4 w = codes_of(stage[wave], i);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc = mfma(read8(w[j], f), x[i][j], acc);
        }
      if (count > PACKED) flush(c0, to);
    }
  }
  if (unit >= 0 && count <= PACKED) flush(0, count);
  __syncthreads();
  auto put = [&](int i, float s) __attribute__((always_inline)) {
    const int n = n0 + (i & 15);
    if (n >= a.d) return;
    const int64_t o = (int64_t)(i >> 4) * a.d + n;
    if (a.out_f32)
      ((float*)a.out)[o] = s;
    else
      ((uint16_t*)a.out)[o] = (uint16_t)pack_bf16(s, 0.f);
  };
  float* const parted = a.part + (int64_t)blockIdx.x / a.splits * a.splits * a.T * 16;
  for (int i = threadIdx.x; i < a.T * 16; i += kDownWaves * 64) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kDownWaves; ++w) s += sums[w * a.T * 16 + i];
    if (a.splits == 1)
      put(i, s);
    else
      store_dev(parted + split * a.T * 16 + i, s);
  }
  if (a.splits == 1) return;
  // the last of the workgroups adds up what they left (every one ends; none waits)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0)
    done = __hip_atomic_fetch_add(&a.counter[blockIdx.x / a.splits], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (done != a.splits - 1) return;
  for (int i = threadIdx.x; i < a.T * 16; i += kDownWaves * 64) {
    float s = 0.f;
    for (int w = 0; w < a.splits; ++w) s += load_dev(parted + w * a.T * 16 + i);
    put(i, s);
  }
}

}  // namespace

// Workgroups of a column tile of the second launch: so many that every compute unit has
// one, but no more than leave a wavefront a batch (both launches, 4 tokens on 128 experts of
// 768 x 2048: 27.6 us on 256 workgroups, 30.0 on 128, 31.5 on 512; 61 tokens: 97, 134, 106).
void few_plan(FewArgs& a) {
  const int cols = (a.d + 15) / 16;
  const int64_t steps = (int64_t)a.units * ((a.f + 127) / 128), most = (steps + kDownWaves * kBatch - 1) / (kDownWaves * kBatch);
  a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({most, 256 / cols, 8}));
  a.counters = a.splits > 1 ? cols : 0;
}

hipError_t launch_few_up(const FewArgs& a, hipStream_t s) {
  const dim3 grid(LX_MX4_KP(a.f) / 16, a.units);  // (in one dimension its threads can pass 32 bits)
  if (a.x_f32)
    k_few_up<true><<<grid, 256, 0, s>>>(a);
  else
    k_few_up<false><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_few_down(const FewArgs& a, hipStream_t s) {
  // next to the codes' 64 KB the sums and the units take up to 88 KB
  static DeviceOnce once;
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e == hipSuccess)
    e = once.run(device, hipSuccess, [] {
      return hipFuncSetAttribute((const void*)k_few_down, hipFuncAttributeMaxDynamicSharedMemorySize,
                                 LX_MOE_FEW_MAX_T * (kDownWaves * 16 * (int)sizeof(float) + LX_MAX_K * 12));
    });
  if (e != hipSuccess) return e;
  const unsigned grid = (unsigned)((a.d + 15) / 16) * a.splits;
  const size_t lds = a.units * 12 + (size_t)kDownWaves * a.T * 16 * sizeof(float);
  k_few_down<<<grid, kDownWaves * 64, lds, s>>>(a);
  return hipGetLastError();
}

}  // namespace lx
