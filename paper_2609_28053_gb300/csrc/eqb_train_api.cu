// eqb_train_api.cu -- the exported entry points of a router's training step
// (declared in include/eqb.h): argument checks, then the launches.
#include <math.h>

#include "eqb_checks.h"

namespace {

// The projection's sizes (eqb_router_logits).
inline eqb_status check_projection(int64_t T, int32_t d, int32_t E) {
  if (T < 0 || d < 1 || E < 1) return EQB_ERR_INVALID_ARG;
  if (d % 64 != 0 || E % 16 != 0 || E > 256) return EQB_ERR_UNSUPPORTED;
  if (T > (int64_t(1) << 31) - (int64_t(1) << 24)) return EQB_ERR_UNSUPPORTED;
  return EQB_OK;
}

inline int64_t valid_bytes(int32_t M) { return static_cast<int64_t>(eqb::carve_round(static_cast<size_t>(M) * 4)); }

}  // namespace

extern "C" {

size_t eqb_balance_loss_workspace_bytes(int64_t T, int32_t E, int32_t M) {
  if (T < 0 || E < 1 || M < 1) return 0;
  return eqb::balance_part_bytes(E, M) + static_cast<size_t>(valid_bytes(M));
}

eqb_status eqb_balance_loss(const void* z, int32_t z_fp32, const int32_t* topk_idx, int64_t T, int32_t E, int32_t K,
                            const int64_t* mb_offsets, int32_t M, const uint8_t* mask, int32_t score, double alpha,
                            double zeta, const float* grad_in, void* grad_out, int32_t grad_out_bf16,
                            const float* grad_scale, int32_t* counts, float* prob, float* loss, void* workspace,
                            size_t workspace_bytes, int32_t* err_flag, void* stream) {
  eqb_status st = check_shape(T, E, K, true);
  if (st != EQB_OK) return st;
  // the factors are used in fp32: infinite there, they would turn a zero into NaN
  if (M < 1 || score < 0 || score > 1 || !isfinite(static_cast<float>(alpha)) || !isfinite(2.0f * static_cast<float>(zeta)) ||
      (score == 1 && zeta != 0.0))
    return EQB_ERR_INVALID_ARG;
  if (M > (1 << 20)) return EQB_ERR_UNSUPPORTED;
  if (!mb_offsets || !counts) return EQB_ERR_INVALID_ARG;
  if (T > 0 && (!topk_idx || (!z && (prob || loss || grad_out)))) return EQB_ERR_INVALID_ARG;
  if (grad_in && !grad_out) return EQB_ERR_INVALID_ARG;
  if (grad_out_bf16 && grad_out && grad_out == static_cast<const void*>(grad_in)) return EQB_ERR_INVALID_ARG;
  if (!aligned(z, 16) || !aligned(topk_idx, 4) || !aligned(mb_offsets, 8) || !aligned(grad_in, 16) || !aligned(grad_out, 16) ||
      !aligned(grad_scale, 4) || !aligned(counts, 4) || !aligned(prob, 4) || !aligned(loss, 4) || !aligned(err_flag, 4))
    return EQB_ERR_INVALID_ARG;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  if (prob || loss || mask) {
    if (!ws || !aligned(ws, 256) || workspace_bytes < eqb_balance_loss_workspace_bytes(T, E, M)) return EQB_ERR_INVALID_ARG;
  }
  eqb::BalanceArgs a{z, z_fp32 != 0, topk_idx, T, E, K, mb_offsets, M, mask, score, alpha, zeta, grad_in, grad_out,
                     grad_out_bf16 != 0, grad_scale, counts, prob, loss,
                     ws ? reinterpret_cast<float*>(ws + valid_bytes(M)) : nullptr, E + 4, reinterpret_cast<int32_t*>(ws),
                     err_flag};
  return to_status(eqb::launch_balance(a, as_stream(stream)));
}

size_t eqb_router_grad_workspace_bytes(int64_t T, int32_t d, int32_t E) {
  if (check_projection(T, d, E) != EQB_OK || T == 0) return 0;
  return eqb::router_grad_workspace(T, d, E);
}

eqb_status eqb_router_grad(const eqb_bf16* dz, const eqb_bf16* x, const eqb_bf16* W_r, int64_t T, int32_t d, int32_t E,
                           eqb_bf16* dx, int32_t accumulate_dx, float* dW, int32_t accumulate_dW, void* workspace,
                           size_t workspace_bytes, int32_t* err_flag, void* stream) {
  eqb_status st = check_projection(T, d, E);
  if (st != EQB_OK) return st;
  if (!aligned(dz, 16) || !aligned(x, 16) || !aligned(W_r, 16) || !aligned(dx, 16) || !aligned(dW, 16) || !aligned(err_flag, 4))
    return EQB_ERR_INVALID_ARG;
  if (T > 0 && (!dz || (dx && !W_r) || (dW && !x))) return EQB_ERR_INVALID_ARG;
  const size_t need = dW ? eqb_router_grad_workspace_bytes(T, d, E) : 0;
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return EQB_ERR_INVALID_ARG;
  if (!dW && (!dx || T == 0)) return EQB_OK;
  eqb::RouterGradArgs a{dz, x, W_r, T, d, E, dx, accumulate_dx != 0, dW, accumulate_dW != 0, static_cast<float*>(workspace),
                        err_flag};
  return to_status(eqb::launch_router_grad(a, as_stream(stream)));
}

eqb_status eqb_adamw_step(const eqb_adamw_tensor* tensors, int32_t count, int32_t state_bits, double lr, int64_t step,
                          double beta1, double beta2, double eps, double weight_decay, const float* grad_scale,
                          int32_t* err_flag, void* stream) {
  if (count < 0 || (count > 0 && !tensors) || (state_bits != 8 && state_bits != 32)) return EQB_ERR_INVALID_ARG;
  if (!(lr >= 0.0) || !isfinite(lr) || step < 1 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) ||
      !(weight_decay >= 0.0) || !isfinite(weight_decay))
    return EQB_ERR_INVALID_ARG;
  // eps alone is the denominator where m = v = 0: it has to be a normal number in fp32
  if (!isnormal(static_cast<float>(eps)) || !(eps > 0.0)) return EQB_ERR_INVALID_ARG;
  if (!aligned(grad_scale, 4) || !aligned(err_flag, 4)) return EQB_ERR_INVALID_ARG;
  const bool bits8 = state_bits == 8;
  for (int32_t i = 0; i < count; ++i) {
    const eqb_adamw_tensor& t = tensors[i];
    if (t.n < 0 || t.n > (int64_t(1) << 40)) return EQB_ERR_INVALID_ARG;
    if (t.n == 0 || !t.grad) continue;
    if (!t.param || !t.exp_avg || !t.exp_avg_sq || (bits8 && (!t.avg_scale || !t.sq_scale)) || (t.copy && t.param_bf16))
      return EQB_ERR_INVALID_ARG;
    if (!aligned(t.param, t.param_bf16 ? 2 : 4) || !aligned(t.grad, t.grad_bf16 ? 2 : 4) || !aligned(t.copy, 2) ||
        !aligned(t.avg_scale, 4) || !aligned(t.sq_scale, 4) ||
        (!bits8 && (!aligned(t.exp_avg, 4) || !aligned(t.exp_avg_sq, 4))))
      return EQB_ERR_INVALID_ARG;
  }
  eqb::AdamwScalars sc;
  sc.b1 = static_cast<float>(beta1);
  sc.c1 = static_cast<float>(1.0 - beta1);
  sc.b2 = static_cast<float>(beta2);
  sc.c2 = static_cast<float>(1.0 - beta2);
  sc.rbc2 = static_cast<float>(1.0 / sqrt(1.0 - pow(beta2, static_cast<double>(step))));
  sc.eps = static_cast<float>(eps);
  sc.decay = static_cast<float>(1.0 - lr * weight_decay);
  sc.step = static_cast<float>(lr / (1.0 - pow(beta1, static_cast<double>(step))));
  if (!isfinite(sc.decay) || !isfinite(sc.step)) return EQB_ERR_INVALID_ARG;
  sc.grad_scale = grad_scale;
  sc.err = err_flag;
  constexpr int kBatch = eqb::kAdamwBatch;
  eqb::AdamwTensor batch[kBatch];
  int n = 0;
  for (int32_t i = 0; i < count; ++i) {
    const eqb_adamw_tensor& t = tensors[i];
    if (t.n > 0 && t.grad) {
      const bool wide = aligned(t.param, 16) && aligned(t.grad, 16) && aligned(t.exp_avg, 16) && aligned(t.exp_avg_sq, 16) &&
                        aligned(t.copy, 16);
      batch[n++] = eqb::AdamwTensor{t.param, t.grad, t.exp_avg, t.exp_avg_sq, t.avg_scale, t.sq_scale, t.copy, t.n,
                                    (t.param_bf16 ? 1 : 0) | (t.grad_bf16 ? 2 : 0) | (wide ? 4 : 0)};
    }
    if (n == kBatch || (i == count - 1 && n > 0)) {
      if (int rc = eqb::launch_adamw(batch, n, state_bits, sc, as_stream(stream))) return to_status(rc);
      n = 0;
    }
  }
  return EQB_OK;
}

}  // extern "C"
