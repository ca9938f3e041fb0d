// C entry points of the operators around the expert layer: argument checks and
// launches. Nothing here allocates or throws.
#include "lx_block.h"

namespace lx {
namespace {

bool al(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool dtype_ok(lx_dtype t) { return t == LX_F32 || t == LX_BF16; }

template <class Args>
lx_status run(const char* name, hipError_t (*fn)(const Args&, hipStream_t), const Args& a, void* stream) {
  struct Call {
    hipError_t (*fn)(const Args&, hipStream_t);
    const Args* a;
  } c{fn, &a};
  const hipError_t e = launch_timed(
      name, (hipStream_t)stream,
      [](const void* p, hipStream_t s) {
        const Call& q = *(const Call*)p;
        return q.fn(*q.a, s);
      },
      &c);
  return e == hipSuccess ? LX_OK : set_error(LX_ERR_HIP, name, hipGetErrorString(e));
}

lx_status check_norm(const lx_norm_layer* p, int32_t T, bool block) {
  if (!p) return set_error(LX_ERR_INVALID_ARGUMENT, "layer is null");
  if (T < 0 || p->d < 1) return set_error(LX_ERR_INVALID_ARGUMENT, "T must be >= 0 and d positive");
  if (p->d % 8 || p->d > LX_NORM_MAX_D) return set_error(LX_ERR_UNSUPPORTED, "d must be a multiple of 8, at most LX_NORM_MAX_D");
  if (!dtype_ok(p->h_dtype) || !dtype_ok(p->y_dtype) || !dtype_ok(p->x_dtype) || !dtype_ok(p->w_dtype))
    return set_error(LX_ERR_INVALID_ARGUMENT, "bad dtype");
  if (!(p->eps >= 0.f)) return set_error(LX_ERR_INVALID_ARGUMENT, "eps must be >= 0");
  if (!al(p->w_pre, 16) || (block && (!al(p->w_post, 16) || !al(p->scale, 16) || !al(p->gate, 4))))
    return set_error(LX_ERR_INVALID_ARGUMENT, "misaligned weight or gate pointer");
  return LX_OK;
}

template <class A>
void norm_layer_args(A& a, const lx_norm_layer& p, int32_t T, bool block) {
  a.T = T;
  a.d = p.d;
  a.h_f32 = p.h_dtype == LX_F32;
  a.y_f32 = p.y_dtype == LX_F32;
  a.x_f32 = p.x_dtype == LX_F32;
  a.w_f32 = p.w_dtype == LX_F32;
  a.alpha = p.residual_scale;
  a.eps = p.eps;
  a.w_pre = p.w_pre;
  a.w_post = block ? p.w_post : nullptr;
  a.scale = block ? p.scale : nullptr;
  a.gate = block ? p.gate : nullptr;
}

lx_status check_balance(lx_dtype dtype, int32_t T, int32_t E, int32_t k) {
  if (T < 0) return set_error(LX_ERR_INVALID_ARGUMENT, "T must be >= 0");
  if (!dtype_ok(dtype)) return set_error(LX_ERR_INVALID_ARGUMENT, "bad dtype");
  if (E < 1 || E > kBalanceMaxE) return set_error(LX_ERR_UNSUPPORTED, "E must be in 1 .. 1024");
  if (k < 1 || k > LX_MAX_K) return set_error(LX_ERR_INVALID_ARGUMENT, "k must be in 1 .. LX_MAX_K");
  if ((int64_t)T * k >= ((int64_t)1 << 31)) return set_error(LX_ERR_UNSUPPORTED, "T * k must be below 2^31");
  return LX_OK;
}

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

struct BalancePlan {
  int blocks;
  size_t part_c, part_n, total;
};
BalancePlan balance_plan(int T, int E) {
  BalancePlan p{};
  p.blocks = balance_blocks(T, E);
  p.part_c = up256((size_t)p.blocks * E * 4);
  p.part_n = p.part_c + up256((size_t)p.blocks * E * 4);
  p.total = p.blocks > 1 ? p.part_n + up256((size_t)p.blocks * 4) : 0;
  return p;
}

lx_status check_mx4(int64_t rows, int32_t K) {
  if (rows < 0 || K < 1) return set_error(LX_ERR_INVALID_ARGUMENT, "rows must be >= 0 and K positive");
  if (K % 8 || K > (1 << 28)) return set_error(LX_ERR_UNSUPPORTED, "K must be a multiple of 8, at most 2^28");
  if (rows > ((int64_t)1 << 40) / LX_MX4_KP(K)) return set_error(LX_ERR_UNSUPPORTED, "rows * K must be below 2^40");
  return LX_OK;
}

lx_status check_mx4_gemm(int32_t M, int32_t N, int32_t K, int32_t G) {
  if (M < 0 || N < 1 || K < 1 || G < 1) return set_error(LX_ERR_INVALID_ARGUMENT, "M must be >= 0; N, K and G positive");
  if (K % 8 || K > (1 << 24)) return set_error(LX_ERR_UNSUPPORTED, "K must be a multiple of 8, at most 2^24");
  if (G > LX_MAX_NODES) return set_error(LX_ERR_UNSUPPORTED, "more groups than LX_MAX_NODES");
  // (rows and columns are counted in 32 bits, up to a tile past the last one)
  if (M > INT32_MAX - 255 || N > INT32_MAX - 255) return set_error(LX_ERR_UNSUPPORTED, "M and N must be at most 2^31 - 256");
  if ((int64_t)M * N >= ((int64_t)1 << 40)) return set_error(LX_ERR_UNSUPPORTED, "M * N must be below 2^40");
  return LX_OK;
}

size_t mx4_gemm_bytes(const Mx4GemmPlan& p, int M, int N) {
  return p.splits > 1 ? up256((size_t)p.splits * M * N * sizeof(float)) : 0;
}

}  // namespace
}  // namespace lx

using namespace lx;

extern "C" {

lx_status lx_block_norm(const lx_norm_layer* layer, int32_t T, const void* h, const void* y, int32_t y_rows,
                        int32_t k, const int32_t* slot_row, const float* slot_weights, void* h_out, void* x,
                        void* stream) {
  clear_error();
  const lx_status st = check_norm(layer, T, y != nullptr);
  if (st != LX_OK) return st;
  if (!slot_row != !slot_weights) return set_error(LX_ERR_INVALID_ARGUMENT, "slot_row and slot_weights: both or neither");
  if (slot_row && (k < 1 || k > LX_MAX_K || y_rows < 0))
    return set_error(LX_ERR_INVALID_ARGUMENT, "k must be in 1 .. LX_MAX_K and y_rows >= 0");
  if (slot_row && (int64_t)T * k >= ((int64_t)1 << 31)) return set_error(LX_ERR_UNSUPPORTED, "T * k must be below 2^31");
  if (!y && (slot_row || h_out)) return set_error(LX_ERR_INVALID_ARGUMENT, "slots and h_out need y");
  if (T == 0) return LX_OK;
  if (!y && !layer->w_pre) return set_error(LX_ERR_INVALID_ARGUMENT, "neither y nor w_pre is given");
  if (!h || (y && !h_out) || !x != !layer->w_pre || !al(h, 16) || !al(y, 16) || !al(h_out, 16) || !al(x, 16) ||
      !al(slot_row, 4) || !al(slot_weights, 4))
    return set_error(LX_ERR_INVALID_ARGUMENT, "null or misaligned pointer");
  NormArgs a{};
  norm_layer_args(a, *layer, T, y != nullptr);
  a.h = h;
  a.y = y;
  a.y_rows = y_rows;
  a.k = slot_row ? k : 0;
  a.slot_row = slot_row;
  a.slot_weights = slot_weights;
  a.h_out = h_out;
  a.x = x;
  return run("block_norm", launch_block_norm, a, stream);
}

size_t lx_block_norm_backward_workspace_bytes(int32_t T, int32_t d) {
  clear_error();
  if (T < 0 || d < 1 || d % 8 || d > LX_NORM_MAX_D) {
    set_error(LX_ERR_INVALID_ARGUMENT, "T must be >= 0, d a multiple of 8 in 8 .. LX_NORM_MAX_D");
    return 0;
  }
  return up256((size_t)norm_grad_groups(T, d) * 2 * d * sizeof(float));
}

lx_status lx_block_norm_backward(const lx_norm_layer* layer, int32_t T, const void* h_out, const void* y,
                                 const void* dx, const void* dh_out, void* dh, void* dy, float* dgate,
                                 float* dw_pre, float* dw_post, float* dscale, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  clear_error();
  const lx_status st = check_norm(layer, T, y != nullptr);
  if (st != LX_OK) return st;
  const lx_norm_layer& p = *layer;
  if (!y && !p.w_pre) return set_error(LX_ERR_INVALID_ARGUMENT, "neither y nor w_pre is given");
  if (!dw_pre != !p.w_pre || !dw_post != !(y && p.w_post) || !dscale != !(y && p.scale))
    return set_error(LX_ERR_INVALID_ARGUMENT, "dw_pre, dw_post and dscale go with w_pre, w_post and scale");
  if (!al(dw_pre, 16) || !al(dw_post, 16) || !al(dscale, 16))
    return set_error(LX_ERR_INVALID_ARGUMENT, "misaligned pointer");
  if (T > 0) {
    if (!h_out || !dh || !dx != !p.w_pre || !dy != !y || !dgate != !(y && p.gate) || !al(h_out, 16) || !al(y, 16) ||
        !al(dx, 16) || !al(dh_out, 16) || !al(dh, 16) || !al(dy, 16) || !al(dgate, 4))
      return set_error(LX_ERR_INVALID_ARGUMENT, "null, superfluous or misaligned pointer");
  }
  if (!workspace || !al(workspace, 256)) return set_error(LX_ERR_INVALID_ARGUMENT, "workspace null or not 256-byte aligned");
  NormGradArgs a{};
  a.groups = norm_grad_groups(T, p.d);
  if (workspace_bytes < up256((size_t)a.groups * 2 * p.d * sizeof(float)))
    return set_error(LX_ERR_WORKSPACE_TOO_SMALL, "workspace smaller than required");
  norm_layer_args(a, p, T, y != nullptr);
  a.h_out = h_out;
  a.y = y;
  a.dx = dx;
  a.dh_out = dh_out;
  a.dh = dh;
  a.dy = dy;
  a.dgate = dgate;
  a.dw_pre = dw_pre;
  a.dw_post = dw_post;
  a.dscale = dscale;
  a.part = (float*)workspace;
  if (T == 0) a.groups = 0;
  if (T > 0) {
    const lx_status s1 = run("block_norm_grad", launch_block_norm_grad, a, stream);
    if (s1 != LX_OK) return s1;
  }
  if (!dw_pre && !dw_post && !dscale) return LX_OK;
  return run("block_norm_grad_sum", launch_block_norm_grad_sum, a, stream);
}

size_t lx_balance_loss_workspace_bytes(int32_t T, int32_t E) {
  clear_error();
  if (check_balance(LX_F32, T, E, 1) != LX_OK) return 0;
  return balance_plan(T, E).total;
}

lx_status lx_balance_loss(const void* logits, lx_dtype dtype, int32_t T, int32_t E, const int32_t* topk_ids,
                          int32_t k, const uint8_t* mask, float coef, float* loss, int32_t* counts, float* prob,
                          int32_t* n_tokens, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const lx_status st = check_balance(dtype, T, E, k);
  if (st != LX_OK) return st;
  if (!loss || !counts || !prob || !n_tokens || !al(loss, 4) || !al(counts, 4) || !al(prob, 4) || !al(n_tokens, 4) ||
      (T > 0 && (!logits || !topk_ids || !al(logits, 16) || !al(topk_ids, 4))))
    return set_error(LX_ERR_INVALID_ARGUMENT, "null or misaligned pointer");
  const BalancePlan P = balance_plan(T, E);
  if (P.total) {
    if (!workspace || !al(workspace, 256)) return set_error(LX_ERR_INVALID_ARGUMENT, "workspace null or not 256-byte aligned");
    if (workspace_bytes < P.total) return set_error(LX_ERR_WORKSPACE_TOO_SMALL, "workspace smaller than required");
  }
  BalanceArgs a{};
  a.T = T;
  a.E = E;
  a.k = k;
  a.f32 = dtype == LX_F32;
  a.coef = coef;
  a.logits = logits;
  a.ids = topk_ids;
  a.mask = mask;
  a.loss = loss;
  a.counts = counts;
  a.prob = prob;
  a.n_tokens = n_tokens;
  a.blocks = P.blocks;
  if (P.total) {
    a.part_p = (float*)workspace;
    a.part_c = (int32_t*)((uint8_t*)workspace + P.part_c);
    a.part_n = (int32_t*)((uint8_t*)workspace + P.part_n);
  }
  const lx_status s1 = run("balance", launch_balance, a, stream);
  if (s1 != LX_OK || P.blocks == 1) return s1;
  return run("balance_sum", launch_balance_sum, a, stream);
}

lx_status lx_balance_loss_backward(const void* logits, lx_dtype dtype, int32_t T, int32_t E, int32_t k,
                                   const uint8_t* mask, const int32_t* counts, const int32_t* n_tokens, float coef,
                                   const float* dloss, void* dlogits, void* stream) {
  clear_error();
  const lx_status st = check_balance(dtype, T, E, k);
  if (st != LX_OK) return st;
  if (T == 0) return LX_OK;
  if (!logits || !counts || !n_tokens || !dlogits || !al(logits, 16) || !al(dlogits, 16) || !al(counts, 4) ||
      !al(n_tokens, 4) || !al(dloss, 4))
    return set_error(LX_ERR_INVALID_ARGUMENT, "null or misaligned pointer");
  BalanceArgs a{};
  a.T = T;
  a.E = E;
  a.k = k;
  a.f32 = dtype == LX_F32;
  a.coef = coef;
  a.logits = logits;
  a.mask = mask;
  a.counts = (int32_t*)counts;
  a.n_tokens = (int32_t*)n_tokens;
  a.dloss = dloss;
  a.dlogits = dlogits;
  return run("balance_grad", launch_balance_grad, a, stream);
}

lx_status lx_mx4_quantize(const void* x, lx_dtype dtype, int64_t rows, int32_t K, lx_mx4_act act, void* codes,
                          void* scales, void* stream) {
  clear_error();
  const lx_status st = check_mx4(rows, K);
  if (st != LX_OK) return st;
  if (!dtype_ok(dtype) || (act != LX_MX4_NONE && act != LX_MX4_SWIGLU))
    return set_error(LX_ERR_INVALID_ARGUMENT, "bad dtype or act");
  if (rows == 0) return LX_OK;
  if (!x || !codes || !scales || !al(x, 16) || !al(codes, 16) || !al(scales, 4))
    return set_error(LX_ERR_INVALID_ARGUMENT, "null or misaligned pointer");
  Mx4Args a{};
  a.x = x;
  a.rows = rows;
  a.K = K;
  a.f32 = dtype == LX_F32;
  a.swiglu = act == LX_MX4_SWIGLU;
  a.codes = (uint8_t*)codes;
  a.scales = (uint8_t*)scales;
  return run("mx4_quantize", launch_mx4_quantize, a, stream);
}

lx_status lx_mx4_dequantize(const void* codes, const void* scales, int64_t rows, int32_t K, void* out,
                            lx_dtype dtype, void* stream) {
  clear_error();
  const lx_status st = check_mx4(rows, K);
  if (st != LX_OK) return st;
  if (!dtype_ok(dtype)) return set_error(LX_ERR_INVALID_ARGUMENT, "bad dtype");
  if (rows == 0) return LX_OK;
  if (!out || !codes || !scales || !al(out, 16) || !al(codes, 16) || !al(scales, 4))
    return set_error(LX_ERR_INVALID_ARGUMENT, "null or misaligned pointer");
  Mx4Args a{};
  a.x = out;
  a.rows = rows;
  a.K = K;
  a.f32 = dtype == LX_F32;
  a.codes = (uint8_t*)codes;
  a.scales = (uint8_t*)scales;
  return run("mx4_dequantize", launch_mx4_dequantize, a, stream);
}

size_t lx_mx4_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t G) {
  clear_error();
  if (check_mx4_gemm(M, N, K, G) != LX_OK) return 0;
  return mx4_gemm_bytes(mx4_gemm_plan(M, N, LX_MX4_KP(K), G), M, N);
}

lx_status lx_mx4_gemm(const void* a, const void* a_scales, int32_t a_rows, const int32_t* row_map, const void* b,
                      const void* b_scales, const int32_t* offsets, int32_t G, int32_t M, int32_t N, int32_t K,
                      void* out, lx_dtype out_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const lx_status st = check_mx4_gemm(M, N, K, G);
  if (st != LX_OK) return st;
  if (!dtype_ok(out_dtype)) return set_error(LX_ERR_INVALID_ARGUMENT, "bad out_dtype");
  if (a_rows < 0 || (!row_map && a_rows < M)) return set_error(LX_ERR_INVALID_ARGUMENT, "a_rows must be >= M without a row map");
  if (!offsets && G != 1) return set_error(LX_ERR_INVALID_ARGUMENT, "several groups need offsets");
  if (M == 0) return LX_OK;
  if (!a || !a_scales || !b || !b_scales || !out || !al(a, 16) || !al(b, 16) || !al(out, 16) || !al(a_scales, 4) ||
      !al(b_scales, 4) || !al(row_map, 4) || !al(offsets, 4))
    return set_error(LX_ERR_INVALID_ARGUMENT, "null or misaligned pointer");
  Mx4GemmArgs g{};
  g.plan = mx4_gemm_plan(M, N, LX_MX4_KP(K), G);
  const size_t need = mx4_gemm_bytes(g.plan, M, N);
  if (need) {
    if (!workspace || !al(workspace, 256)) return set_error(LX_ERR_INVALID_ARGUMENT, "workspace null or not 256-byte aligned");
    if (workspace_bytes < need) return set_error(LX_ERR_WORKSPACE_TOO_SMALL, "workspace smaller than required");
  }
  // the tile kernels address A by 32-bit byte offsets (and a tile's weights, at most
  // 2^31 bytes)
  if (a_rows == 0 || (int64_t)a_rows * (LX_MX4_KP(K) / 2) >= ((int64_t)1 << 32)) g.plan = {Mx4GemmPlan::kRows, 1, 0};
  g.part = (float*)workspace;
  g.a = (const uint8_t*)a;
  g.as = (const uint8_t*)a_scales;
  g.b = (const uint8_t*)b;
  g.bs = (const uint8_t*)b_scales;
  g.a_rows = a_rows;
  g.row_map = row_map;
  g.offsets = offsets;
  g.G = G;
  g.M = M;
  g.N = N;
  g.Kp = LX_MX4_KP(K);
  g.out_f32 = out_dtype == LX_F32;
  g.out = out;
  const lx_status s1 = run("mx4_gemm", launch_mx4_gemm, g, stream);
  if (s1 != LX_OK || g.plan.splits == 1) return s1;
  return run("mx4_gemm_sum", launch_mx4_gemm_sum, g, stream);
}

}  // extern "C"
