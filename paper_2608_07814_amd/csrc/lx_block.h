// Internal declarations of the operators around the expert layer (block norms,
// balance loss, 4-bit values): kernel arguments and launch functions.
#pragma once

#include "lx_internal.h"
#include "lx_philox.h"
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
  Dropout drop;      // of the block's output (rng null: none)
};
// Whether the forward has its lean form (lx_norm_rows.h).
inline bool norm_lean(const NormArgs& a) { return !a.h_f32 && !a.w_f32 && !(a.y && a.y_f32) && !a.slot_row; }
hipError_t launch_block_norm(const NormArgs& a, hipStream_t s);
// The same with x in 8 bits too (x itself null: only these).
struct Norm8Args : NormArgs {
  uint8_t *x_codes, *x_scales;
};
hipError_t launch_block_norm_mx8(const Norm8Args& a, hipStream_t s);

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
  Dropout drop;      // as in the forward
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
// The same with 8-bit values (LX_MX8_KP codes of a byte a row).
hipError_t launch_mx8_quantize(const Mx4Args& a, hipStream_t s);
hipError_t launch_mx8_dequantize(const Mx4Args& a, hipStream_t s);

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

// Products of 8-bit activations and 4-bit weights.
struct Mx8GemmPlan {
  enum Kernel : int32_t { kRows, kRows4, kTile64, kTile128, kTile256 } kernel;
  bool tile() const { return kernel >= kTile64; }
};
// rows_only: the tile kernels cannot run.
Mx8GemmPlan mx8_gemm_plan(int M, int N, int Kp, int G, bool swiglu, bool rows_only);
struct Mx8GemmArgs {
  const uint8_t *a, *as, *b, *bs;
  int32_t a_rows;
  const int32_t* row_map;
  const int32_t* offsets;
  int32_t G, M, N, Kp;
  int32_t cols;          // of the result: N, N / 2 with SwiGLU
  int32_t act;
  const void *bias, *res;
  uint8_t bias_f32, res_f32, out_f32;
  void* out;
  uint8_t* out_scales;   // not null: the result is in 8 bits
  Mx8GemmPlan plan;
};
hipError_t launch_mx8_gemm(const Mx8GemmArgs& a, hipStream_t s);

// ------------------------------------------------------------ a layer for a few tokens
struct FewUnit {
  int32_t expert, base;
  uint64_t mask;
};
struct FewArgs {
  const void* x;
  int32_t T, k, E, d, f;
  uint8_t x_f32, out_f32;
  const int32_t* ids;
  const float* weights;
  const uint8_t *gu, *gu_s, *down, *down_s;
  void* out;
  int32_t units;         // min(E, T k): the experts, or the slots
  int32_t splits, counters;  // few_plan
  // left by the first launch for the second, per unit: its expert (-1: it has no
  // tokens), the first of its rows of hidden, and its tokens as bits
  FewUnit* unit;         // [units]
  uint16_t* hidden;      // [T k][3][LX_MX4_KP(f)]: bf16 terms
  int32_t* counter;      // [counters], cleared by the first launch
  float* part;           // splits > 1: [d / 16][splits][T][16]
};
// From d, f and units the split of the work.
void few_plan(FewArgs& a);
hipError_t launch_few_up(const FewArgs& a, hipStream_t s);
hipError_t launch_few_down(const FewArgs& a, hipStream_t s);

}  // namespace lx
