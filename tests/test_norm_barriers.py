"""Every thread of a workgroup of the norm kernels reaches as many barriers, for
whatever number of rows the last round has: the kernels compiled for the CPU, their
threads run one after the other, with barriers counted and lane exchanges left
out (no result is looked at)."""
import os
import subprocess

from paper_2608_07814_amd import build as B

RUNTIME = """
#pragma once
#include <cmath>
#include <cstdint>
#include <cstring>
#include <algorithm>
using std::max;
using std::min;
#define __global__
#define __device__
#define __host__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __restrict__
struct Dim { int x = 0, y = 0, z = 0; };
inline Dim threadIdx, blockIdx, gridDim;
inline int barriers;
inline void __syncthreads() { ++barriers; }
inline float __uint_as_float(uint32_t x) { float f; memcpy(&f, &x, 4); return f; }
inline uint32_t __float_as_uint(float f) { uint32_t x; memcpy(&x, &f, 4); return x; }
struct Two { uint32_t v[2]; uint32_t operator[](int i) const { return v[i]; } };
#define __builtin_amdgcn_update_dpp(old, x, ...) (x)
#define __builtin_amdgcn_readfirstlane(x) ((int)(x))
#define __builtin_amdgcn_fmed3f(a, b, c) ((a) + (b) + (c))
#define __builtin_amdgcn_permlane16_swap(a, b, ...) (Two{{(a), (b)}})
#define __builtin_amdgcn_permlane32_swap(a, b, ...) (Two{{(a), (b)}})
typedef void* hipStream_t;
typedef int hipError_t;
"""

MAIN = """
extern "C" __bf16 __truncsfbf2(float x) {
  const uint16_t h = __float_as_uint(x) >> 16;
  return __builtin_bit_cast(__bf16, h);
}
#include <cstdio>
#include <vector>
using namespace lx;

// The kernel on `grid` workgroups of `threads`: 0 if all threads of each reach as
// many barriers, else the workgroup's number + 1.
template <class K, class A>
int uneven(K kernel, const A& a, int grid, int threads) {
  gridDim.x = grid;
  for (int b = 0; b < grid; ++b) {
    int first = 0;
    for (int t = 0; t < threads; ++t) {
      blockIdx.x = b;
      threadIdx.x = t;
      barriers = 0;
      kernel(a);
      if (t == 0) first = barriers;
      if (barriers != first) return b + 1;
    }
  }
  return 0;
}

template <int TPR, int NV>
void check(int d) {
  for (int grid : {1, 2})
    for (int T = 1; T <= 7; ++T)
      for (int parts = 0; parts < 4; ++parts) {
        std::vector<uint16_t> h((size_t)T * d), y(h), x(h), o(h), w(d);
        NormArgs a{};
        a.T = T;
        a.d = d;
        a.alpha = 1;
        a.eps = 1e-6f;
        a.h = h.data();
        a.y = y.data();
        a.h_out = o.data();
        a.x = x.data();
        a.w_pre = parts & 1 ? w.data() : nullptr;
        a.w_post = parts & 2 ? w.data() : nullptr;
        if (int b = uneven(k_block_norm<TPR, NV>, a, grid, kFwdThreads<TPR>))
          std::printf("forward d=%d T=%d parts=%d: workgroup %d of %d\\n", d, T, parts, b - 1, grid);
        std::vector<float> part((size_t)grid * 2 * d), gate(T);
        NormGradArgs g{};
        g.T = T;
        g.d = d;
        g.alpha = 1;
        g.eps = 1e-6f;
        g.h_out = h.data();
        g.y = y.data();
        g.dh_out = x.data();
        g.dh = o.data();
        g.dy = y.data();
        g.dx = parts & 1 ? x.data() : nullptr;
        g.w_pre = a.w_pre;
        g.w_post = a.w_post;
        g.part = part.data();
        g.groups = grid;
        if (int b = uneven(k_block_norm_grad<true, TPR, NV, NV == 1>, g, grid, kBwd))
          std::printf("backward d=%d T=%d parts=%d: workgroup %d of %d\\n", d, T, parts, b - 1, grid);
      }
}

int main() {
  check<64, 1>(64);
  check<128, 1>(520);
  check<256, 1>(1032);
  check<512, 1>(2056);
  check<1024, 2>(8200);
}
"""


def test_every_thread_reaches_every_barrier(tmp_path):
    source = open(os.path.join(B.CSRC, "k_norm.hip")).read()
    kernels, launches = source.split("template <class F>\nhipError_t by_width", 1)
    assert "__global__" not in launches
    (tmp_path / "hip").mkdir()
    (tmp_path / "hip" / "hip_runtime.h").write_text(RUNTIME)
    header = open(os.path.join(B.CSRC, "lx_block.h")).read()
    (tmp_path / "lx_block.h").write_text(header.replace('#include "lx_internal.h"', "#include <hip/hip_runtime.h>"))
    kernels = kernels.replace('asm volatile("" : "+v"', 'asm volatile("" : "+m"')
    kernels = kernels.replace('"+v"(r.b)', '"+m"(r.b)')
    (tmp_path / "norm.cpp").write_text(kernels + "}  // namespace\n}  // namespace lx\n" + MAIN)
    exe = str(tmp_path / "norm")
    subprocess.run([os.path.join(os.path.dirname(B.HIPCC), "amdclang++"), "-std=c++17", "-O1", "-w", "-I", str(tmp_path), "-I", B.CSRC,
                    "-I", B.INCLUDE, str(tmp_path / "norm.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], check=True, stdout=subprocess.PIPE, text=True).stdout
    assert not out, out
