// eqb_expert_api.cu -- the exported entry points of the experts behind a router
// (declared in include/eqb.h): argument checks, then the launches.
#include <math.h>

#include "eqb_checks.h"

namespace {

constexpr int64_t kMaxRows = (int64_t(1) << 31) - (int64_t(1) << 24);  // 32-bit row numbers need headroom
constexpr int kMaxWidth = 1 << 20;

// A width that the 8-bit operands come in.
inline eqb_status check_width(int32_t d) {
  if (d < 1) return EQB_ERR_INVALID_ARG;
  return d % 16 != 0 || d > kMaxWidth ? EQB_ERR_UNSUPPORTED : EQB_OK;
}
inline eqb_status check_rows(int64_t n) {
  if (n < 0) return EQB_ERR_INVALID_ARG;
  return n > kMaxRows ? EQB_ERR_UNSUPPORTED : EQB_OK;
}
// T lists of K entries.
inline eqb_status check_lists(int64_t T, int32_t K) {
  if (T < 0 || K < 1) return EQB_ERR_INVALID_ARG;
  return K > 1024 || T > kMaxRows / K ? EQB_ERR_UNSUPPORTED : EQB_OK;
}
inline eqb_status check_experts(int32_t E) {
  if (E < 1) return EQB_ERR_INVALID_ARG;
  return E > eqb::kMaxExperts ? EQB_ERR_UNSUPPORTED : EQB_OK;
}
inline eqb_status worst(eqb_status a, eqb_status b) { return a != EQB_OK ? a : b; }

}  // namespace

extern "C" {

eqb_status eqb_gate_topk(const void* z, int32_t z_fp32, const float* b, int64_t T, int32_t E, int32_t K, int32_t groups,
                         int32_t top_groups, int32_t group_top2, int32_t score, int32_t renorm, double scale,
                         const uint8_t* mask, int32_t* topk_idx, float* weight, int32_t* err_flag, void* stream) {
  eqb_status st = check_shape(T, E, K, true);
  if (st != EQB_OK) return st;
  if (groups < 1 || top_groups < 1 || top_groups > groups || E % groups != 0 || K > top_groups * (E / groups) || score < 0 ||
      score > 1 || !isfinite(static_cast<float>(scale)))
    return EQB_ERR_INVALID_ARG;
  if (groups > 32) return EQB_ERR_UNSUPPORTED;
  if (T > 0 && (!z || !topk_idx)) return EQB_ERR_INVALID_ARG;
  if (!aligned(z, 16) || !aligned(b, 4) || !aligned(topk_idx, 4) || !aligned(weight, 4) || !aligned(err_flag, 4))
    return EQB_ERR_INVALID_ARG;
  if (T == 0) return EQB_OK;
  eqb::GateArgs a{z, z_fp32 != 0, b, T, E, K, groups, top_groups, group_top2 != 0, score, renorm != 0, static_cast<float>(scale),
                  mask, topk_idx, weight, err_flag};
  return to_status(eqb::launch_gate(a, as_stream(stream)));
}

eqb_status eqb_gate_grad(const void* z, int32_t z_fp32, const int32_t* topk_idx, const float* grad_weight, int64_t T, int32_t E,
                         int32_t K, int32_t score, int32_t renorm, double scale, const float* grad_in, void* grad_out,
                         int32_t grad_out_bf16, void* stream) {
  eqb_status st = check_shape(T, E, K, true);
  if (st != EQB_OK) return st;
  if (score < 0 || score > 1 || !isfinite(static_cast<float>(scale))) return EQB_ERR_INVALID_ARG;
  if (T > 0 && (!z || !topk_idx || !grad_weight || !grad_out)) return EQB_ERR_INVALID_ARG;
  if (grad_out_bf16 && grad_out && grad_out == static_cast<const void*>(grad_in)) return EQB_ERR_INVALID_ARG;
  if (!aligned(z, 16) || !aligned(topk_idx, 4) || !aligned(grad_weight, 4) || !aligned(grad_in, 16) || !aligned(grad_out, 16))
    return EQB_ERR_INVALID_ARG;
  if (T == 0) return EQB_OK;
  eqb::GateGradArgs a{z, z_fp32 != 0, topk_idx, grad_weight, T, E, K, score, renorm != 0, static_cast<float>(scale), grad_in,
                      grad_out, grad_out_bf16 != 0};
  return to_status(eqb::launch_gate_grad(a, as_stream(stream)));
}

size_t eqb_expert_rows_workspace_bytes(int64_t T, int32_t K, int32_t E) {
  if (worst(check_lists(T, K), check_experts(E)) != EQB_OK) return 0;
  return eqb::expert_rows_workspace(T * K, E);
}

eqb_status eqb_expert_rows(const int32_t* topk_idx, int64_t T, int32_t K, int32_t E, int32_t* offsets, int32_t* blocks,
                           int32_t* slot, int32_t* entry, void* workspace, size_t workspace_bytes, void* stream) {
  const eqb_status st = worst(check_lists(T, K), check_experts(E));
  if (st != EQB_OK) return st;
  if (!offsets || !blocks || (T > 0 && (!topk_idx || !slot || !entry))) return EQB_ERR_INVALID_ARG;
  if (!aligned(topk_idx, 4) || !aligned(offsets, 4) || !aligned(blocks, 4) || !aligned(slot, 4) || !aligned(entry, 4))
    return EQB_ERR_INVALID_ARG;
  const size_t need = eqb_expert_rows_workspace_bytes(T, K, E);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return EQB_ERR_INVALID_ARG;
  eqb::ExpertRowsArgs a{topk_idx, T * K, E, offsets, blocks, slot, entry, static_cast<int32_t*>(workspace)};
  return to_status(eqb::launch_expert_rows(a, as_stream(stream)));
}

int64_t eqb_expert_max_blocks(int64_t R, int32_t E) {
  if (R < 0 || E < 1) return -1;
  constexpr int64_t B = eqb::kExpertBlock;
  return (R + (B - 1) * (R < E ? R : E)) / B;
}

eqb_status eqb_quant_rows(const eqb_bf16* x, int64_t T, int32_t d, const int32_t* slot, int32_t K, uint8_t* q, float* scale,
                          int32_t* err_flag, void* stream) {
  eqb_status st = worst(check_width(d), slot ? check_lists(T, K) : check_rows(T));
  if (st != EQB_OK) return st;
  if (T > 0 && (!x || !q || !scale)) return EQB_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(q, 16) || !aligned(scale, 4) || !aligned(slot, 4) || !aligned(err_flag, 4))
    return EQB_ERR_INVALID_ARG;
  if (T == 0) return EQB_OK;
  return to_status(eqb::launch_quant_rows(x, T, d, slot, slot ? K : 1, q, scale, err_flag, as_stream(stream)));
}

eqb_status eqb_quant_cols(const eqb_bf16* x, int64_t T, int32_t c, const int32_t* entry, int64_t R, int32_t K,
                          const int32_t* offsets, const int32_t* blocks, int32_t E, int64_t P, uint8_t* q, float* scale,
                          int32_t* err_flag, void* stream) {
  eqb_status st = worst(worst(check_width(c), check_experts(E)), worst(check_rows(T), check_rows(R)));
  if (st != EQB_OK) return st;
  if (P < 0 || (entry && K < 1) || (!entry && T < R)) return EQB_ERR_INVALID_ARG;
  if (P > kMaxRows / 128) return EQB_ERR_UNSUPPORTED;
  if (!offsets || !blocks || (P > 0 && (!q || !scale)) || (T > 0 && !x)) return EQB_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(entry, 4) || !aligned(offsets, 4) || !aligned(blocks, 4) || !aligned(q, 16) ||
      !aligned(scale, 4) || !aligned(err_flag, 4))
    return EQB_ERR_INVALID_ARG;
  if (P == 0 || R == 0) return EQB_OK;
  eqb::QuantColsArgs a{x, T, c, entry, R, entry ? K : 1, offsets, blocks, E, P, q, scale, err_flag};
  return to_status(eqb::launch_quant_cols(a, as_stream(stream)));
}

eqb_status eqb_quant_blocks(const void* w, int32_t w_fp32, int32_t E, int32_t n, int32_t d, uint8_t* q, float* scale,
                            uint8_t* q_t, float* scale_t, int32_t* err_flag, void* stream) {
  if (E < 0) return EQB_ERR_INVALID_ARG;
  eqb_status st = worst(worst(check_width(n), check_width(d)), E > eqb::kMaxExperts ? EQB_ERR_UNSUPPORTED : EQB_OK);
  if (st != EQB_OK) return st;
  if (E > 0 && (!w || !q || !scale)) return EQB_ERR_INVALID_ARG;
  if ((q_t == nullptr) != (scale_t == nullptr)) return EQB_ERR_INVALID_ARG;
  if (!aligned(w, 16) || !aligned(q, 16) || !aligned(scale, 4) || !aligned(q_t, 16) || !aligned(scale_t, 4) ||
      !aligned(err_flag, 4))
    return EQB_ERR_INVALID_ARG;
  if (E == 0) return EQB_OK;
  return to_status(eqb::launch_quant_blocks(w, w_fp32 != 0, E, n, d, q, scale, q_t, scale_t, err_flag, as_stream(stream)));
}

eqb_status eqb_expert_matmul(const uint8_t* q, const float* scale, const uint8_t* w, const float* w_scale,
                             const int32_t* offsets, int64_t R, int32_t n, int32_t d, int32_t E, void* out, int32_t out_fp32,
                             int32_t* err_flag, void* stream) {
  eqb_status st = worst(worst(check_width(n), check_width(d)), worst(check_experts(E), check_rows(R)));
  if (st != EQB_OK) return st;
  if (!offsets || (R > 0 && (!q || !scale || !w || !w_scale || !out))) return EQB_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(scale, 4) || !aligned(w, 16) || !aligned(w_scale, 4) || !aligned(offsets, 4) ||
      !aligned(out, 32) || !aligned(err_flag, 4))
    return EQB_ERR_INVALID_ARG;
  if (R == 0) return EQB_OK;
  eqb::ExpertMatmulArgs a{q, scale, w, w_scale, offsets, R, n, d, E, out, out_fp32 != 0, 0, err_flag};
  return to_status(eqb::launch_expert_matmul(a, as_stream(stream)));
}

eqb_status eqb_expert_wgrad(const uint8_t* a, const float* a_scale, const uint8_t* b, const float* b_scale,
                            const int32_t* blocks, int64_t P, int32_t n, int32_t d, int32_t E, float* dW, int32_t accumulate,
                            int32_t* err_flag, void* stream) {
  if (P < 0) return EQB_ERR_INVALID_ARG;
  eqb_status st = worst(worst(check_width(n), check_width(d)), worst(check_experts(E), P > kMaxRows / 128 ? EQB_ERR_UNSUPPORTED : EQB_OK));
  if (st != EQB_OK) return st;
  if (!blocks || !dW || (P > 0 && (!a || !a_scale || !b || !b_scale))) return EQB_ERR_INVALID_ARG;
  if (!aligned(a, 16) || !aligned(a_scale, 4) || !aligned(b, 16) || !aligned(b_scale, 16) || !aligned(blocks, 4) ||
      !aligned(dW, 32) || !aligned(err_flag, 4))
    return EQB_ERR_INVALID_ARG;
  if (P == 0 && accumulate) return EQB_OK;
  eqb::ExpertMatmulArgs g{a, a_scale, b, b_scale, blocks, P, n, d, E, dW, 1, accumulate != 0, err_flag};
  return to_status(eqb::launch_expert_wgrad(g, as_stream(stream)));
}

eqb_status eqb_expert_combine(const eqb_bf16* rows, const int32_t* slot, const float* weight, int64_t T, int64_t R, int32_t n,
                              int32_t K, eqb_bf16* out, void* stream) {
  eqb_status st = worst(check_width(n), worst(check_lists(T, K), check_rows(R)));
  if (st != EQB_OK) return st;
  if (T > 0 && (!slot || !out || (R > 0 && !rows))) return EQB_ERR_INVALID_ARG;
  if (!aligned(rows, 16) || !aligned(slot, 4) || !aligned(weight, 4) || !aligned(out, 16)) return EQB_ERR_INVALID_ARG;
  if (T == 0) return EQB_OK;
  eqb::CombineArgs a{nullptr, rows, slot, weight, T, R, n, K, out, nullptr};
  return to_status(eqb::launch_combine(a, as_stream(stream)));
}

eqb_status eqb_expert_combine_grad(const eqb_bf16* grad, const eqb_bf16* rows, const int32_t* slot, const float* weight,
                                   int64_t T, int64_t R, int32_t n, int32_t K, eqb_bf16* grad_rows, float* grad_weight,
                                   void* stream) {
  eqb_status st = worst(check_width(n), worst(check_lists(T, K), check_rows(R)));
  if (st != EQB_OK) return st;
  if (T > 0 && (!slot || !grad || (R > 0 && grad_weight && !rows))) return EQB_ERR_INVALID_ARG;
  if (!aligned(grad, 16) || !aligned(rows, 16) || !aligned(slot, 4) || !aligned(weight, 4) || !aligned(grad_rows, 16) ||
      !aligned(grad_weight, 4))
    return EQB_ERR_INVALID_ARG;
  if (T == 0 || (!grad_rows && !grad_weight)) return EQB_OK;
  eqb::CombineArgs a{grad, rows, slot, weight, T, R, n, K, grad_rows, grad_weight};
  return to_status(eqb::launch_combine_grad(a, as_stream(stream)));
}

}  // extern "C"
