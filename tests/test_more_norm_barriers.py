"""Every thread of a workgroup of the norm kernels with dropout, of their lean forms and
of those with an 8-bit output reaches as many barriers, whatever the last round holds:
compiled for the CPU with the stand-ins of the plain norms' test."""
import os
import subprocess

import pytest

from paper_2608_07814_amd import build as B
from test_norm_barriers import MAIN, RUNTIME

MORE = RUNTIME + """
struct uint2 { uint32_t x, y; };
inline uint2 make_uint2(uint32_t x, uint32_t y) { return {x, y}; }
#define __builtin_amdgcn_cvt_pk_fp8_f32(a, b, old, hi) ((int)((a) + (b)) + (old))
"""

CHECK = MAIN[:MAIN.index("template <int TPR, int NV>")] + """
template <int TPR, int NV>
void check(int d) {
  for (int grid : {1, 2})
    for (int T = 1; T <= 7; ++T)
      for (int parts = 0; parts < 4; ++parts) {
        const int Kp = LX_MX8_KP(d);
        std::vector<uint16_t> h((size_t)T * d), y(h), x(h), o(h), w(d);
        std::vector<uint8_t> codes((size_t)T * Kp), scales((size_t)T * Kp / 32);
        const uint64_t rng[2] = {1, 2};
        ARGS a{};
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
        a.drop = Dropout{rng, 30000, 2.f};
        FORWARD
        BACKWARD
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

SAY = 'std::printf("%s d=%d T=%d parts=%d: workgroup %d of %d\\n", __func__, d, T, parts, b - 1, grid);'
NORM = f"""
        if (int b = uneven(k_block_norm<TPR, NV, true, true>, a, grid, kFwdThreads<TPR>)) {SAY}
        if (int b = uneven(k_block_norm<TPR, NV, true, false>, a, grid, kFwdThreads<TPR>)) {SAY}
        if (int b = uneven(k_block_norm<TPR, NV, false, true>, a, grid, kFwdThreads<TPR>)) {SAY}
"""
GRAD = f"""
        std::vector<float> part((size_t)grid * 2 * d);
        NormGradArgs g{{}};
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
        g.drop = a.drop;
        if (int b = uneven(k_block_norm_grad<true, TPR, NV, NV == 1, true>, g, grid, kBwd)) {SAY}
"""
NORM8 = f"""
        a.x_codes = codes.data();
        a.x_scales = scales.data();
        if (int b = uneven(k_block_norm_mx8<TPR, NV, true>, a, grid, kFwdThreads<TPR>)) {SAY}
        if (int b = uneven(k_block_norm_mx8<TPR, NV, false>, a, grid, kFwdThreads<TPR>)) {SAY}
"""


@pytest.mark.parametrize("src,launches,args,forward,backward", [
    ("k_norm.hip", "template <class F>\nhipError_t by_width", "NormArgs", NORM, GRAD),
    ("k_norm8.hip", "template <int TPR, int NV>\nhipError_t launch", "Norm8Args", NORM8, "")])
def test_every_thread_reaches_every_barrier(tmp_path, src, launches, args, forward, backward):
    kernels, rest = open(os.path.join(B.CSRC, src)).read().split(launches, 1)
    assert "__global__" not in rest
    (tmp_path / "hip").mkdir()
    (tmp_path / "hip" / "hip_runtime.h").write_text(MORE)
    header = open(os.path.join(B.CSRC, "lx_block.h")).read()
    (tmp_path / "lx_block.h").write_text(header.replace('#include "lx_internal.h"', "#include <hip/hip_runtime.h>"))
    kernels = kernels.replace('asm volatile("" : "+v"', 'asm volatile("" : "+m"').replace('"+v"(r.b)', '"+m"(r.b)')
    main = CHECK.replace("ARGS", args).replace("FORWARD", forward).replace("BACKWARD", backward)
    (tmp_path / "norm.cpp").write_text(kernels + "}  // namespace\n}  // namespace lx\n" + main)
    exe = str(tmp_path / "norm")
    subprocess.run([os.path.join(os.path.dirname(B.HIPCC), "amdclang++"), "-std=c++17", "-O1", "-w", "-I", str(tmp_path), "-I", B.CSRC,
                    "-I", B.INCLUDE, str(tmp_path / "norm.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], check=True, stdout=subprocess.PIPE, text=True).stdout
    assert not out, out
