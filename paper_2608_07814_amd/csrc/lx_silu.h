// SwiGLU's activation by the machine's own exponential and reciprocal.
#pragma once

#include <hip/hip_runtime.h>

namespace lx {

// z / (1 + exp(-z)) by the exponential and reciprocal instructions (an ulp each, and
// |z| 2^-24 from the product that is the exponent). Far below 0 the exponential is
// infinite and the result -0.
__device__ __forceinline__ float silu(float z) {
  return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896341f * z));
}

}  // namespace lx
