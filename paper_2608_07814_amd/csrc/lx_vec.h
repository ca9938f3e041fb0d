// Device helpers of the row-wise kernels: 8 consecutive values of fp32 or bf16
// at a time (the type is a uniform run-time flag), and sums over lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lx {

typedef float vf4 __attribute__((ext_vector_type(4)));
typedef uint32_t vu4 __attribute__((ext_vector_type(4)));
typedef __bf16 vb2 __attribute__((ext_vector_type(2)));

struct F8 {
  float v[8];
};

// 8 values as they lie in memory: two (fp32) or one (bf16) 16-byte loads, so
// that many can be in flight before the first is converted.
struct Raw8 {
  vu4 a, b;
};

__device__ __forceinline__ Raw8 load_raw8(const void* p, bool f32, int64_t i) {
  Raw8 r;
  if (f32) {
    const vu4* q = (const vu4*)((const float*)p + i);
    r.a = q[0];
    r.b = q[1];
  } else {
    r.a = *(const vu4*)((const uint16_t*)p + i);
    r.b = r.a;
  }
  return r;
}

__device__ __forceinline__ F8 unpack8(const Raw8& r, bool f32) {
  F8 o;
  if (f32) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o.v[j] = __uint_as_float(r.a[j]);
      o.v[4 + j] = __uint_as_float(r.b[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o.v[2 * j] = __uint_as_float(r.a[j] << 16);
      o.v[2 * j + 1] = __uint_as_float(r.a[j] & 0xFFFF0000u);
    }
  }
  return o;
}

__device__ __forceinline__ F8 load8(const void* p, bool f32, int64_t i) { return unpack8(load_raw8(p, f32, i), f32); }

// The same where the type is known to be bf16.
struct RawB8 {
  vu4 a;
};
template <class R>
__device__ __forceinline__ R load_as(const void* p, bool f32, int64_t i) {
  if constexpr (sizeof(R) == sizeof(RawB8))
    return R{*(const vu4*)((const uint16_t*)p + i)};
  else
    return load_raw8(p, f32, i);
}
__device__ __forceinline__ F8 unpack8(const RawB8& r, bool) { return unpack8(Raw8{r.a, r.a}, false); }

// two values to bf16, round to nearest even
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const vb2 q = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, q);
}

__device__ __forceinline__ void store8(void* p, bool f32, int64_t i, const F8& x) {
  if (f32) {
    vf4* q = (vf4*)((float*)p + i);
    q[0] = vf4{x.v[0], x.v[1], x.v[2], x.v[3]};
    q[1] = vf4{x.v[4], x.v[5], x.v[6], x.v[7]};
  } else {
    *(vu4*)((uint16_t*)p + i) = vu4{pack_bf16(x.v[0], x.v[1]), pack_bf16(x.v[2], x.v[3]), pack_bf16(x.v[4], x.v[5]),
                                    pack_bf16(x.v[6], x.v[7])};
  }
}

// 8 values to a place that is only aligned to its type.
typedef uint32_t vu4h __attribute__((ext_vector_type(4), aligned(2)));
typedef float vf4w __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void store8_any(void* p, bool f32, int64_t i, const F8& x) {
  if (f32) {
    vf4w* q = (vf4w*)((float*)p + i);
    q[0] = vf4w{x.v[0], x.v[1], x.v[2], x.v[3]};
    q[1] = vf4w{x.v[4], x.v[5], x.v[6], x.v[7]};
  } else {
    *(vu4h*)((uint16_t*)p + i) = vu4h{pack_bf16(x.v[0], x.v[1]), pack_bf16(x.v[2], x.v[3]), pack_bf16(x.v[4], x.v[5]),
                                      pack_bf16(x.v[6], x.v[7])};
  }
}

// The value of the lane that DPP control C selects (all lanes active).
template <int C>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), C, 0xF, 0xF, true));
}

// Sum (OP 0) or maximum (OP 1, NaN dropped) over groups of LANES consecutive
// lanes, in every lane of the group: exchanges within 16 lanes are DPP, the
// wider ones swap halves between two copies.
template <int LANES, int OP = 0>
__device__ __forceinline__ float lane_reduce(float x) {
  auto op = [](float a, float b) { return OP ? fmaxf(a, b) : a + b; };
  if constexpr (LANES >= 2) x = op(x, dpp<0xB1>(x));    // quad_perm 1 0 3 2
  if constexpr (LANES >= 4) x = op(x, dpp<0x4E>(x));    // quad_perm 2 3 0 1
  if constexpr (LANES >= 8) x = op(x, dpp<0x141>(x));   // row_half_mirror
  if constexpr (LANES >= 16) x = op(x, dpp<0x140>(x));  // row_mirror
  if constexpr (LANES >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (LANES >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return x;
}
// Sum over the lanes of the wavefront that agree in lane % STRIDE.
template <int STRIDE>
__device__ __forceinline__ float stride_sum(float x) {
  static_assert(STRIDE >= 8 && STRIDE <= 64, "");
  if constexpr (STRIDE <= 8) x += dpp<0x128>(x);  // row_ror:8
  if constexpr (STRIDE <= 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (STRIDE <= 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}
template <int LANES>
__device__ __forceinline__ float lane_sum(float x) {
  return lane_reduce<LANES, 0>(x);
}
template <int LANES>
__device__ __forceinline__ float lane_max(float x) {
  return lane_reduce<LANES, 1>(x);
}

}  // namespace lx
