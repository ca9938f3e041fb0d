// Internal declarations of the operators around the expert layer (block norms,
// balance loss, 4-bit values): kernel arguments and launch functions.
#pragma once

#include "lx_internal.h"
#include "lorex_block.h"

namespace lx {

// ------------------------------------------------------------ host services
// (host.hip) The calling thread's error message; set_error returns `s` and
// never throws, so it may be used at a C entry point.
void clear_error() noexcept;
lx_status set_error(lx_status s, const char* what, const char* detail = nullptr) noexcept;
// Kernel timing records around a launch, as for the forward's kernels.
hipError_t launch_timed(const char* name, hipStream_t s, hipError_t (*launch)(const void*, hipStream_t),
                        const void* args) noexcept;

// ------------------------------------------------------------ block norms
struct NormArgs {
  int32_t T, d, k, y_rows;
  uint8_t h_f32, y_f32, x_f32, w_f32;
  float alpha, eps;
  const void *w_pre, *w_post, *scale;
  const float* gate;
  const void *h, *y;
  const int32_t* slot_row;
  const float* slot_weights;
  void *h_out, *x;
};
hipError_t launch_block_norm(const NormArgs& a, hipStream_t s);

struct NormGradArgs {
  int32_t T, d;
  uint8_t h_f32, y_f32, x_f32, w_f32;
  float alpha, eps;
  const void *w_pre, *w_post, *scale;
  const float* gate;
  const void *h_out, *y, *dx, *dh_out;
  void *dh, *dy;
  float *dgate, *dw_pre, *dw_post, *dscale;
  float* part;       // [groups][2][d]: sums of dx m and of gate D n
  int32_t groups;
};
// Workgroups of the backward, each with its partial weight gradients.
int norm_grad_groups(int T, int d);
hipError_t launch_block_norm_grad(const NormGradArgs& a, hipStream_t s);
hipError_t launch_block_norm_grad_sum(const NormGradArgs& a, hipStream_t s);

// ------------------------------------------------------------ balance loss
constexpr int kBalanceMaxE = 1024;
struct BalanceArgs {
  int32_t T, E, k;
  uint8_t f32;
  float coef;
  const void* logits;
  const int32_t* ids;
  const uint8_t* mask;
  float* loss;
  int32_t* counts;
  float* prob;
  int32_t* n_tokens;
  // forward, more than one workgroup: per workgroup E probability sums, E
  // counts, 1 token count
  float* part_p;
  int32_t* part_c;
  int32_t* part_n;
  int32_t blocks;
  // backward
  const float* dloss;
  void* dlogits;
};
int balance_blocks(int T, int E);
hipError_t launch_balance(const BalanceArgs& a, hipStream_t s);
hipError_t launch_balance_sum(const BalanceArgs& a, hipStream_t s);
hipError_t launch_balance_grad(const BalanceArgs& a, hipStream_t s);

// ------------------------------------------------------------ 4-bit values
struct Mx4Args {
  const void* x;
  int64_t rows;
  int32_t K;
  uint8_t f32, swiglu;
  uint8_t* codes;
  uint8_t* scales;
};
hipError_t launch_mx4_quantize(const Mx4Args& a, hipStream_t s);
// x is the output of the reading back
hipError_t launch_mx4_dequantize(const Mx4Args& a, hipStream_t s);

// Which kernel a product runs on, and into how many parts its K is split (each
// but the last of split_steps steps of 256 values).
struct Mx4GemmPlan {
  enum Kernel : int32_t { kRows, kRows4, kTile64, kTile128, kTile256 } kernel;
  int32_t splits, split_steps;
};
Mx4GemmPlan mx4_gemm_plan(int M, int N, int Kp, int G);
struct Mx4GemmArgs {
  const uint8_t *a, *as, *b, *bs;
  int32_t a_rows;
  const int32_t* row_map;
  const int32_t* offsets;
  int32_t G, M, N, Kp;
  uint8_t out_f32;
  void* out;
  float* part;       // splits > 1: [splits][M][N]
  Mx4GemmPlan plan;
};
hipError_t launch_mx4_gemm(const Mx4GemmArgs& a, hipStream_t s);
hipError_t launch_mx4_gemm_sum(const Mx4GemmArgs& a, hipStream_t s);

}  // namespace lx
