// The block norms with the next block's input in 8 bits (formulas in lorex_block.h):
// the rows of k_norm.hip, whose lanes hold 8 consecutive columns each, so that four
// of them share a block and its scale goes over them by DPP. Bound by memory like
// the norms with a bf16 output, of which this writes half: 8192 x 4096 in bf16 46 us over
// four sets of inputs in turn (236 MB, 5.2 TB/s), 48 to 53 where its result is read back in
// between, 2048 x 8192 27, one row of 2048 with 8 experts' fp32 rows 5.0.
#include "lx_block.h"
#include "lx_mx8.h"
#include "lx_norm_rows.h"

#include <algorithm>

namespace lx {
namespace {

template <int TPR, int NV, bool LEAN>
__global__ __launch_bounds__(kFwdThreads<TPR>) void k_block_norm_mx8(const Norm8Args a) {
  __shared__ float lds[2 * kFwdThreads<TPR> / 64];
  const int Kp = LX_MX8_KP(a.d);
  block_norm_rows<TPR, NV, false, LEAN>(a, lds, [&](int64_t t, int col, bool in, bool live, F8 x) __attribute__((always_inline)) {
    // (past d, where a zero may have met an infinite factor, the row is padded with zeros)
    if (!in) x = F8{};
    if (a.x && in && live) store8(a.x, a.x_f32, t * a.d + col, x);
    int s;
    const uint2 code = mx8_round(x, s);
    if (live && col < Kp) {
      *(uint2*)(a.x_codes + t * Kp + col) = code;
      if ((threadIdx.x & 3) == 0) a.x_scales[t * (Kp / 32) + col / 32] = (uint8_t)s;
    }
  });
}

template <int TPR, int NV>
hipError_t launch(const Norm8Args& a, hipStream_t s) {
  constexpr int THR = kFwdThreads<TPR>, RPB = THR / TPR;
  const int grid = (int)std::min<int64_t>(((int64_t)a.T + RPB - 1) / RPB, 256 * (2048 / THR));
  if (norm_lean(a))
    k_block_norm_mx8<TPR, NV, true><<<grid, THR, 0, s>>>(a);
  else
    k_block_norm_mx8<TPR, NV, false><<<grid, THR, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// A row's lanes hold one group of 8 columns each as long as 1024 lanes do.
hipError_t launch_block_norm_mx8(const Norm8Args& a, hipStream_t s) {
  const int n = LX_MX8_KP(a.d);
  if (n <= 512) return launch<64, 1>(a, s);
  if (n <= 1024) return launch<128, 1>(a, s);
  if (n <= 2048) return launch<256, 1>(a, s);
  if (n <= 4096) return launch<512, 1>(a, s);
  if (n <= 8192) return launch<1024, 1>(a, s);
  if (n <= 16384) return launch<1024, 2>(a, s);
  return launch<1024, 4>(a, s);
}

}  // namespace lx
