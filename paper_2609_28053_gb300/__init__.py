"""GB300-native EQB + LEI routing-balance path (arXiv 2609.28053).

Thin Python binding over the C ABI of ``libeqb.so`` (include/eqb.h).  Each
function has the C entry point's name, checks dtypes/devices/shapes, and
passes raw device pointers plus the current CUDA stream; every step of the
path runs in the library's CUDA kernels.  PyTorch provides device memory
and streams only.

The routing-balance step of one MoE layer, in the paper's order:

    eqb_route_topk        Sec. 2: top-K of z + b, cutoff tau_t, loads f_e
                          (+ Algorithm 1 step 1, the coarse histogram)
    eqb_select_quantile   Algorithm 1 step 3 (pass 1): u_e, rho_e
    eqb_margin_hist_pass2 Algorithm 1 step 4: fine histogram
    eqb_select_quantile   Algorithm 1 steps 5-6 (pass 2): exact quantile
    eqb_bias_update       Eq. (2): centred bias for the next step
    lei_inject_grad       Sec. 4: Eq. (LEI) with Eq. (norm)

and, for layers whose logits are produced here, eqb_router_logits (Sec. 2,
z_t = W_r x_t) on the tensor cores.
"""
from __future__ import annotations

import ctypes
from array import array

import torch
from torch.autograd.graph import increment_version

from ._lib import STATUS, AdamwTensor, EqbError, load

__all__ = [
    "EqbError", "STATUS", "load", "eqb_target_rank", "eqb_route_topk", "eqb_margin_hist_pass1",
    "eqb_margin_hist_pass2", "eqb_select_quantile", "eqb_bias_update", "lei_inject_grad",
    "EqbWorkspace", "eqb_layer_forward", "eqb_router_logits", "eqb_layer_workspace_bytes",
    "eqb_layer_step", "eqb_layer_step_noalloc", "eqb_router_route", "eqb_router_layer_step",
    "eqb_maxvio", "gshard_inject_grad", "eqb_rank_averaged_bias", "eqb_fixed_hist_bias",
    "eqb_rank_averaged_workspace_bytes", "eqb_selftest_stalled_wait", "lei_coefficients",
    "eqb_margin_hist_lei", "eqb_balance_loss", "eqb_balance_loss_workspace_bytes", "eqb_router_grad",
    "eqb_router_grad_workspace_bytes", "EqbAdamW", "eqb_gate_topk", "eqb_gate_grad", "eqb_expert_rows",
    "eqb_expert_rows_workspace_bytes", "eqb_expert_max_blocks", "eqb_quant_rows", "eqb_quant_cols", "eqb_quant_blocks",
    "eqb_expert_matmul", "eqb_expert_wgrad", "eqb_expert_combine", "eqb_expert_combine_grad",
]


def _p(t):
    return None if t is None else t.data_ptr()


# torch's own shortcuts to the raw handle of the current stream (a stream object
# takes longer to make than a small call to launch); they are private, so a
# release without them falls back to the public call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    """The raw stream handle; the current stream of the current device by
    default (the tensors of a call are on the GPU, so CUDA is initialised)."""
    if stream is None:
        if _raw_stream is not None and _raw_device is not None:
            return _raw_stream(_raw_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _new(shape, dtype, like, stream, make=torch.empty):
    """A tensor that a call makes itself, on the device of `like`.  It comes from
    the memory of the stream that the call launches on: torch hands a freed block
    to the next request of the stream it was taken on, in that stream's order, so
    memory of another one may still be in use when the call's kernels start, or be
    in use again before they end."""
    if stream is None:
        return make(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype, device=like.device)


def _need(t, dtype, name, shape=None):
    # one line for a tensor that fits, the reasons below for one that does not:
    # a call checks up to ten tensors, which takes longer than its launches
    if t is None or (type(t) is torch.Tensor and t.dtype is dtype and t.is_cuda and t.is_contiguous()
                     and (shape is None or t.shape == shape)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _on_current_device(t, name):
    """The library takes its scratch and streams from the CUDA device that is
    current when it is called: the tensors must live on that device."""
    cur = torch.cuda.current_device()
    if t.device.index != cur:
        raise ValueError(f"{name} is on cuda:{t.device.index} but cuda:{cur} is the current device; "
                         f"call inside torch.cuda.device({t.device})")


def _check(rc, what):
    if rc != 0:
        raise EqbError(rc, what)


def eqb_target_rank(T: int, E: int, K: int) -> int:
    return int(load().eqb_target_rank(T, E, K))


def eqb_route_topk(z, b, K, mb_offsets=None, topk_idx=None, tau=None, loads=None, hist_hi=None,
                   err_flag=None, stream=None):
    """Top-K routing, cutoffs and loads (+ optional coarse histogram).
    z bf16 [T,E]; b fp32 [E]; mb_offsets int64 [M+1]; outputs as in eqb.h.
    loads and hist_hi are accumulated into.  Returns (topk_idx, tau)."""
    T, E = z.shape
    _need(z, torch.bfloat16, "z")
    _need(b, torch.float32, "b", (E,))
    if tau is None:
        tau = _new(T, torch.float32, z, stream)
    _need(tau, torch.float32, "tau", (T,))
    _need(topk_idx, torch.int32, "topk_idx", (T, K))
    M = 0
    if mb_offsets is not None:
        _need(mb_offsets, torch.int64, "mb_offsets")
        M = mb_offsets.numel() - 1
    _need(loads, torch.int32, "loads", (M, E) if loads is not None else None)
    _need(hist_hi, torch.int32, "hist_hi", (E, 256))
    _need(err_flag, torch.int32, "err_flag")
    rc = load().eqb_route_topk(_p(z), _p(b), T, E, K, _p(mb_offsets), M, _p(topk_idx), _p(tau),
                               _p(loads), _p(hist_hi), _p(err_flag), _stream(stream))
    _check(rc, "eqb_route_topk")
    return topk_idx, tau


def eqb_route_hist_fused(z, b, K, mb_offsets=None, topk_idx=None, tau=None, loads=None, hist_hi=None,
                         err_flag=None, stream=None):
    """Routing and the coarse histogram from one kernel that reads z once
    (E = 128 or 256): the outputs of eqb_route_topk with hist_hi, bit for
    bit.  Returns tau."""
    T, E = z.shape
    _need(z, torch.bfloat16, "z")
    _need(b, torch.float32, "b", (E,))
    if tau is None:
        tau = _new(T, torch.float32, z, stream)
    _need(tau, torch.float32, "tau", (T,))
    _need(topk_idx, torch.int32, "topk_idx", (T, K))
    _need(mb_offsets, torch.int64, "mb_offsets")
    M = 0 if mb_offsets is None else mb_offsets.numel() - 1
    _need(loads, torch.int32, "loads", (M, E) if loads is not None else None)
    _need(hist_hi, torch.int32, "hist_hi", (E, 256))
    if hist_hi is None:
        raise ValueError("hist_hi is required")
    _need(err_flag, torch.int32, "err_flag")
    _check(load().eqb_route_hist_fused(_p(z), _p(b), T, E, int(K), _p(mb_offsets), M, _p(topk_idx), _p(tau),
                                       _p(loads), _p(hist_hi), _p(err_flag), _stream(stream)),
           "eqb_route_hist_fused")
    return tau


def eqb_margin_hist_pass1(z, tau, hist_hi, err_flag=None, stream=None):
    T, E = z.shape
    _need(z, torch.bfloat16, "z")
    _need(tau, torch.float32, "tau", (T,))
    _need(hist_hi, torch.int32, "hist_hi", (E, 256))
    _need(err_flag, torch.int32, "err_flag")
    _check(load().eqb_margin_hist_pass1(_p(z), _p(tau), T, E, _p(hist_hi), _p(err_flag),
                                        _stream(stream)), "eqb_margin_hist_pass1")


def eqb_margin_hist_pass2(z, tau, u, hist_lo, stream=None):
    T, E = z.shape
    _need(z, torch.bfloat16, "z")
    _need(tau, torch.float32, "tau", (T,))
    _need(u, torch.uint8, "u", (E,))
    _need(hist_lo, torch.int32, "hist_lo", (E, 256))
    _check(load().eqb_margin_hist_pass2(_p(z), _p(tau), T, E, _p(u), _p(hist_lo), _stream(stream)),
           "eqb_margin_hist_pass2")


def eqb_select_quantile(hist, pass_, r, u, rho, q_hat=None, err_flag=None, stream=None):
    E = hist.shape[0]
    _need(hist, torch.int32, "hist", (E, 256))
    _need(u, torch.uint8, "u", (E,))
    _need(rho, torch.int32, "rho", (E,))
    _need(q_hat, torch.bfloat16, "q_hat", (E,))
    _need(err_flag, torch.int32, "err_flag")
    _check(load().eqb_select_quantile(_p(hist), E, int(pass_), int(r), _p(u), _p(rho), _p(q_hat),
                                      _p(err_flag), _stream(stream)), "eqb_select_quantile")


def eqb_bias_update(q_hat, b_next, stream=None):
    E = q_hat.shape[0]
    _need(q_hat, torch.bfloat16, "q_hat", (E,))
    _need(b_next, torch.float32, "b_next", (E,))
    _check(load().eqb_bias_update(_p(q_hat), E, _p(b_next), _stream(stream)), "eqb_bias_update")


def lei_inject_grad(grad_s, loads, mb_offsets, K, eta, c, stream=None):
    T, E = grad_s.shape
    _need(grad_s, torch.float32, "grad_s")
    _need(mb_offsets, torch.int64, "mb_offsets")
    M = mb_offsets.numel() - 1
    _need(loads, torch.int32, "loads", (M, E))
    _check(load().lei_inject_grad(_p(grad_s), _p(loads), _p(mb_offsets), M, T, E, K, float(eta),
                                  float(c), _stream(stream)), "lei_inject_grad")


def lei_coefficients(loads, mb_offsets, K, eta, c, coef=None, stream=None):
    """The [M,E] table of LEI coefficients eta * sigma_l * rho_{l,e} (the
    values lei_inject_grad adds).  Returns coef (fp32 [M,E])."""
    M, E = loads.shape
    _need(loads, torch.int32, "loads")
    _need(mb_offsets, torch.int64, "mb_offsets", (M + 1,))
    if coef is None:
        coef = _new((M, E), torch.float32, loads, stream)
    _need(coef, torch.float32, "coef", (M, E))
    _check(load().lei_coefficients(_p(loads), _p(mb_offsets), M, E, int(K), float(eta), float(c), _p(coef),
                                   _stream(stream)), "lei_coefficients")
    return coef


def eqb_margin_hist_lei(z, tau, pass_, hist, grad_s, coef, mb_offsets, lei_t0, lei_t1, u=None,
                        err_flag=None, stream=None):
    """A histogram pass (1: coarse, 2: fine, needs u) with grad_s[t] +=
    coef[mb(t)] for t in [lei_t0, lei_t1) streamed beside it, one kernel."""
    T, E = z.shape
    _need(z, torch.bfloat16, "z")
    _need(tau, torch.float32, "tau", (T,))
    _need(hist, torch.int32, "hist", (E, 256))
    _need(u, torch.uint8, "u", (E,))
    _need(err_flag, torch.int32, "err_flag")
    _need(grad_s, torch.float32, "grad_s", (T, E))
    _need(mb_offsets, torch.int64, "mb_offsets")
    M = mb_offsets.numel() - 1
    _need(coef, torch.float32, "coef", (M, E))
    _check(load().eqb_margin_hist_lei(_p(z), _p(tau), T, E, int(pass_), _p(u), _p(hist), _p(err_flag),
                                      _p(grad_s), _p(coef), _p(mb_offsets), M, int(lei_t0), int(lei_t1),
                                      _stream(stream)), "eqb_margin_hist_lei")


def eqb_router_logits(x, W_r, z=None, err_flag=None, stream=None):
    """Router logits z = bf16(x W_r^T), fp32 accumulation on the tensor cores.
    x bf16 [T,d], W_r bf16 [E,d]; returns z bf16 [T,E]."""
    T, d = x.shape
    E = W_r.shape[0]
    _need(x, torch.bfloat16, "x")
    _need(W_r, torch.bfloat16, "W_r", (E, d))
    if z is None:
        z = _new((T, E), torch.bfloat16, x, stream)
    _need(z, torch.bfloat16, "z", (T, E))
    _need(err_flag, torch.int32, "err_flag")
    _check(load().eqb_router_logits(_p(x), _p(W_r), T, d, E, _p(z), _p(err_flag), _stream(stream)),
           "eqb_router_logits")
    return z


def eqb_router_route(x, W_r, b, K, mb_offsets=None, z=None, topk_idx=None, tau=None, loads=None,
                     err_flag=None, stream=None, hist_hi=None):
    """Router logits and routing in one kernel (see eqb.h): z = bf16(x W_r^T)
    and, from the same accumulators, eqb_route_topk's topk_idx, tau and loads
    (accumulated into); with hist_hi [E,256] also the coarse histogram
    (accumulated into).  E in {64, 128}, K <= 8.  Returns (z, topk_idx, tau)."""
    T, d = x.shape
    E = W_r.shape[0]
    _need(x, torch.bfloat16, "x")
    _need(W_r, torch.bfloat16, "W_r", (E, d))
    _need(b, torch.float32, "b", (E,))
    if z is None:
        z = _new((T, E), torch.bfloat16, x, stream)
    if tau is None:
        tau = _new(T, torch.float32, x, stream)
    _need(z, torch.bfloat16, "z", (T, E))
    _need(tau, torch.float32, "tau", (T,))
    _need(topk_idx, torch.int32, "topk_idx", (T, K))
    M = 0
    if mb_offsets is not None:
        _need(mb_offsets, torch.int64, "mb_offsets")
        M = mb_offsets.numel() - 1
    _need(loads, torch.int32, "loads", (M, E) if loads is not None else None)
    _need(hist_hi, torch.int32, "hist_hi", (E, 256) if hist_hi is not None else None)
    _need(err_flag, torch.int32, "err_flag")
    _check(load().eqb_router_route(_p(x), _p(W_r), T, d, E, K, _p(b), _p(mb_offsets), M, _p(z),
                                   _p(topk_idx), _p(tau), _p(loads), _p(hist_hi), _p(err_flag), _stream(stream)),
           "eqb_router_route")
    return z, topk_idx, tau


def gshard_inject_grad(grad_s, z, loads, mb_offsets, K, alpha, stream=None):
    """GShard auxiliary-loss gradient added to grad_s in place (see eqb.h):
    grad_s fp32 [T,E], z bf16 [T,E], loads int32 [M,E], mb_offsets int64."""
    T, E = z.shape
    _need(grad_s, torch.float32, "grad_s", (T, E))
    _need(z, torch.bfloat16, "z")
    _need(mb_offsets, torch.int64, "mb_offsets")
    M = mb_offsets.numel() - 1
    _need(loads, torch.int32, "loads", (M, E))
    _check(load().gshard_inject_grad(_p(grad_s), _p(z), _p(loads), _p(mb_offsets), M, T, E, K,
                                     float(alpha), _stream(stream)), "gshard_inject_grad")
    return grad_s


def eqb_rank_averaged_workspace_bytes(E: int, P: int) -> int:
    return int(load().eqb_rank_averaged_workspace_bytes(E, P))


def eqb_rank_averaged_bias(z, tau, K, shard_offsets_host, workspace, b_out=None, q_shards=None,
                           err_flag=None, stream=None):
    """Rank-averaged QB (Sec. 2): each shard's own K/E margin quantile,
    averaged over the non-empty shards and centered.  shard_offsets_host: int64
    host array [P+1]; workspace: uint8 CUDA tensor of
    eqb_rank_averaged_workspace_bytes(E, P) bytes.  Returns (b fp32 [E],
    q_shards bf16 [P,E], row p = shard p)."""
    import numpy as np
    T, E = z.shape
    _need(z, torch.bfloat16, "z")
    _need(tau, torch.float32, "tau", (T,))
    off = np.ascontiguousarray(np.asarray(shard_offsets_host), dtype=np.int64)
    P = len(off) - 1
    if b_out is None:
        b_out = _new(E, torch.float32, z, stream)
    if q_shards is None:
        q_shards = _new((P, E), torch.bfloat16, z, stream, torch.zeros)
    _need(b_out, torch.float32, "b_out", (E,))
    _need(q_shards, torch.bfloat16, "q_shards", (P, E))
    _need(workspace, torch.uint8, "workspace")
    _need(err_flag, torch.int32, "err_flag")
    _check(load().eqb_rank_averaged_bias(_p(z), _p(tau), T, E, K, off.ctypes.data_as(ctypes.c_void_p), P,
                                         _p(q_shards), _p(b_out), _p(workspace), workspace.numel(),
                                         _p(err_flag), _stream(stream)), "eqb_rank_averaged_bias")
    return b_out, q_shards


def eqb_fixed_hist_bias(z, tau, K, lo, width, workspace, b_out=None, estimate=None, err_flag=None,
                        stream=None):
    """Fixed-resolution (256 equal bins) histogram estimate of the K/E margin
    quantile (Sec. 2), centered.  Returns (b fp32 [E], estimate fp64 [E])."""
    T, E = z.shape
    _need(z, torch.bfloat16, "z")
    _need(tau, torch.float32, "tau", (T,))
    if b_out is None:
        b_out = _new(E, torch.float32, z, stream)
    if estimate is None:
        estimate = _new(E, torch.float64, z, stream)
    _need(b_out, torch.float32, "b_out", (E,))
    _need(estimate, torch.float64, "estimate", (E,))
    _need(workspace, torch.uint8, "workspace")
    _need(err_flag, torch.int32, "err_flag")
    _check(load().eqb_fixed_hist_bias(_p(z), _p(tau), T, E, K, float(lo), float(width), _p(b_out),
                                      _p(estimate), _p(workspace), workspace.numel(), _p(err_flag),
                                      _stream(stream)), "eqb_fixed_hist_bias")
    return b_out, estimate


def eqb_selftest_stalled_wait(err_flag, polls=1 << 16, stream=None):
    """Run the bounded-wait failure path on purpose (see eqb.h): afterwards
    err_flag holds EQB_ERR_CUDA and the context is still usable."""
    _need(err_flag, torch.int32, "err_flag")
    _check(load().eqb_selftest_stalled_wait(_p(err_flag), int(polls), _stream(stream)),
           "eqb_selftest_stalled_wait")


def eqb_maxvio(loads, mb_offsets, K, out=None, per_mb=None, stream=None):
    """Global and Local MaxVio (Sec. 5 metrics) of int32 loads [M,E] over the
    microbatches given by mb_offsets; returns a float64 CUDA tensor [2]
    (global, local)."""
    M, E = loads.shape
    _need(loads, torch.int32, "loads")
    _need(mb_offsets, torch.int64, "mb_offsets", (M + 1,))
    if out is None:
        out = _new(2, torch.float64, loads, stream)
    _need(out, torch.float64, "out", (2,))
    _need(per_mb, torch.float64, "per_mb", (M,) if per_mb is not None else None)
    _check(load().eqb_maxvio(_p(loads), _p(mb_offsets), M, E, K, _p(out), _p(per_mb), _stream(stream)),
           "eqb_maxvio")
    return out


def eqb_layer_workspace_bytes(E: int) -> int:
    return int(load().eqb_layer_workspace_bytes(E))


def eqb_layer_step(z, b, K, mb_offsets, loads, b_next, workspace, tau=None, topk_idx=None,
                   grad_s=None, eta=0.0, c=0.0, mb_offsets_host=None, r=0, err_flag=None,
                   stream=None):
    """The whole routing-balance step of one layer in one library call (see
    eqb.h).  workspace: uint8 CUDA tensor of eqb_layer_workspace_bytes(E)
    bytes.  mb_offsets_host: optional int64 host copy of the offsets, checked
    by the library before anything is launched."""
    T, E = z.shape
    _need(z, torch.bfloat16, "z")
    _need(b, torch.float32, "b", (E,))
    _need(mb_offsets, torch.int64, "mb_offsets")
    M = mb_offsets.numel() - 1
    _need(loads, torch.int32, "loads", (M, E))
    _need(b_next, torch.float32, "b_next", (E,))
    _need(workspace, torch.uint8, "workspace")
    if tau is None:
        tau = _new(T, torch.float32, z, stream)
    _need(tau, torch.float32, "tau", (T,))
    _need(topk_idx, torch.int32, "topk_idx", (T, K))
    _need(grad_s, torch.float32, "grad_s", (T, E) if grad_s is not None else None)
    _need(err_flag, torch.int32, "err_flag")
    host = None
    if mb_offsets_host is not None:
        import numpy as np
        host = np.ascontiguousarray(np.asarray(mb_offsets_host), dtype=np.int64)
        if host.shape != (M + 1,):
            raise ValueError("mb_offsets_host must have M+1 entries")
    hp = None if host is None else host.ctypes.data_as(ctypes.c_void_p)
    rc = load().eqb_layer_step(_p(z), _p(b), T, E, K, _p(mb_offsets), hp, M, int(r), _p(topk_idx),
                               _p(tau), _p(loads), _p(b_next), _p(grad_s), float(eta), float(c),
                               _p(workspace), workspace.numel(), _p(err_flag), _stream(stream))
    _check(rc, "eqb_layer_step")
    return tau


def eqb_router_layer_step(x, W_r, b, K, mb_offsets, loads, b_next, workspace, z=None, tau=None,
                          topk_idx=None, grad_s=None, eta=0.0, c=0.0, mb_offsets_host=None, r=0,
                          err_flag=None, stream=None):
    """The routing-balance step of one layer from the router input x (see
    eqb.h): the projection z = bf16(x W_r^T), routed from its accumulators
    where the shape allows, then everything eqb_layer_step does.  Returns
    (z, tau)."""
    T, d = x.shape
    E = W_r.shape[0]
    _need(x, torch.bfloat16, "x")
    _need(W_r, torch.bfloat16, "W_r", (E, d))
    _need(b, torch.float32, "b", (E,))
    _need(mb_offsets, torch.int64, "mb_offsets")
    M = mb_offsets.numel() - 1
    _need(loads, torch.int32, "loads", (M, E))
    _need(b_next, torch.float32, "b_next", (E,))
    _need(workspace, torch.uint8, "workspace")
    if z is None:
        z = _new((T, E), torch.bfloat16, x, stream)
    if tau is None:
        tau = _new(T, torch.float32, x, stream)
    _need(z, torch.bfloat16, "z", (T, E))
    _need(tau, torch.float32, "tau", (T,))
    _need(topk_idx, torch.int32, "topk_idx", (T, K))
    _need(grad_s, torch.float32, "grad_s", (T, E) if grad_s is not None else None)
    _need(err_flag, torch.int32, "err_flag")
    host = None
    if mb_offsets_host is not None:
        import numpy as np
        host = np.ascontiguousarray(np.asarray(mb_offsets_host), dtype=np.int64)
        if host.shape != (M + 1,):
            raise ValueError("mb_offsets_host must have M+1 entries")
    hp = None if host is None else host.ctypes.data_as(ctypes.c_void_p)
    rc = load().eqb_router_layer_step(_p(x), _p(W_r), T, d, E, K, _p(b), _p(mb_offsets), hp, M, int(r),
                                      _p(z), _p(topk_idx), _p(tau), _p(loads), _p(b_next), _p(grad_s),
                                      float(eta), float(c), _p(workspace), workspace.numel(),
                                      _p(err_flag), _stream(stream))
    _check(rc, "eqb_router_layer_step")
    return z, tau


def eqb_layer_step_noalloc(z, b, K, mb_offsets, loads, b_next, tau=None, topk_idx=None,
                           grad_s=None, eta=0.0, c=0.0, mb_offsets_host=None, r=0, err_flag=None,
                           stream=None):
    """eqb_layer_step without a workspace argument, for callers that cannot
    allocate device memory: the step's scratch is an array inside the
    library (E <= 256).  Calls that overlap on the GPU share that array and
    race; the first call on a device should come before any stream capture.
    z (and every other tensor) must be on the current CUDA device: the
    library looks the scratch array up on that device."""
    T, E = z.shape
    _need(z, torch.bfloat16, "z")
    _on_current_device(z, "z")
    _need(b, torch.float32, "b", (E,))
    _need(mb_offsets, torch.int64, "mb_offsets")
    M = mb_offsets.numel() - 1
    _need(loads, torch.int32, "loads", (M, E))
    _need(b_next, torch.float32, "b_next", (E,))
    if tau is None:
        tau = _new(T, torch.float32, z, stream)
    _need(tau, torch.float32, "tau", (T,))
    _need(topk_idx, torch.int32, "topk_idx", (T, K))
    _need(grad_s, torch.float32, "grad_s", (T, E) if grad_s is not None else None)
    _need(err_flag, torch.int32, "err_flag")
    hp = None
    if mb_offsets_host is not None:
        import numpy as np
        host = np.ascontiguousarray(np.asarray(mb_offsets_host), dtype=np.int64)
        if host.shape != (M + 1,):
            raise ValueError("mb_offsets_host must have M+1 entries")
        hp = host.ctypes.data_as(ctypes.c_void_p)
    rc = load().eqb_layer_step_noalloc(_p(z), _p(b), T, E, K, _p(mb_offsets), hp, M, int(r),
                                       _p(topk_idx), _p(tau), _p(loads), _p(b_next), _p(grad_s),
                                       float(eta), float(c), _p(err_flag), _stream(stream))
    _check(rc, "eqb_layer_step_noalloc")
    return tau


class EqbWorkspace:
    """Device buffers of one layer's EQB statistic: the two [E,256] int32
    histograms, u, rho, q_hat and the error word.  Allocated once by the
    caller (through torch), reused every step."""

    def __init__(self, E: int, device="cuda"):
        self.E = E
        # what zero_() clears lies in one buffer: one fill in place of three
        self._cleared = torch.zeros(2 * E * 256 + 1, dtype=torch.int32, device=device)
        self.hist_hi = self._cleared[:E * 256].view(E, 256)
        self.hist_lo = self._cleared[E * 256:2 * E * 256].view(E, 256)
        self.err = self._cleared[2 * E * 256:]
        self.u = torch.zeros(E, dtype=torch.uint8, device=device)
        self.rho = torch.zeros(E, dtype=torch.int32, device=device)
        self.q_hat = torch.zeros(E, dtype=torch.bfloat16, device=device)

    def zero_(self):
        self._cleared.zero_()
        for t in (self.hist_hi, self.hist_lo, self.err):
            if t._base is not self._cleared:  # replaced by the caller
                t.zero_()


def eqb_layer_forward(z, b, K, mb_offsets, ws: EqbWorkspace, topk_idx, tau, loads, b_next,
                      r=None, stream=None):
    """One layer's forward routing-balance statistic, in the paper's order:
    routing + coarse pass, select 1, fine pass, select 2, bias update.
    `loads` must be zeroed by the caller (it is accumulated into); the
    workspace histograms are zeroed here.  All steps run on `stream`."""
    T, E = z.shape
    if r is None:
        r = eqb_target_rank(T, E, K)
    if stream is None:
        ws.zero_()
    else:
        with torch.cuda.stream(stream):
            ws.zero_()
    eqb_route_topk(z, b, K, mb_offsets, topk_idx, tau, loads, ws.hist_hi, ws.err, stream)
    eqb_select_quantile(ws.hist_hi, 1, r, ws.u, ws.rho, None, ws.err, stream)
    eqb_margin_hist_pass2(z, tau, ws.u, ws.hist_lo, stream)
    eqb_select_quantile(ws.hist_lo, 2, r, ws.u, ws.rho, ws.q_hat, ws.err, stream)
    eqb_bias_update(ws.q_hat, b_next, stream)


def eqb_balance_loss_workspace_bytes(T: int, E: int, M: int) -> int:
    return int(load().eqb_balance_loss_workspace_bytes(T, E, M))


_SCORES = {"softmax": 0, "sigmoid": 1}


def eqb_balance_loss(z, topk_idx, mb_offsets, alpha, zeta=0.0, score="softmax", mask=None, grad_in=None, grad_out=None,
                     grad_scale=None, counts=None, prob=None, loss=None, workspace=None, err_flag=None, stream=None):
    """Balance loss, z-loss and per-expert counts of every microbatch, and
    their gradient, from one pass over z (see eqb.h).  z bf16 or fp32 [T,E];
    topk_idx int32 [T,K]; mask bool or uint8 [T].  With grad_out (fp32 or bf16
    [T,E]) the gradient is written as grad_in + grad_scale * d, or without
    grad_in as grad_scale * d; grad_out may be grad_in.  grad_in is dL/dz: the
    path's grad_s, dL/ds of s = sigmoid(z), is multiplied by s (1 - s) before it
    is given here.  prob (fp32 [M,E])
    takes the mean probabilities when given.  Returns (loss fp32 [M,2]: balance
    loss and z-loss; counts int32 [M,E])."""
    T, E = z.shape
    fp32 = z.dtype is torch.float32
    _need(z, torch.float32 if fp32 else torch.bfloat16, "z")
    _on_current_device(z, "z")
    K = topk_idx.shape[1] if topk_idx.dim() == 2 else 0
    _need(topk_idx, torch.int32, "topk_idx", (T, K))
    _need(mb_offsets, torch.int64, "mb_offsets")
    M = mb_offsets.numel() - 1
    kind = _SCORES.get(score)
    if kind is None:
        raise ValueError(f"score must be one of {sorted(_SCORES)}, got {score!r}")
    if mask is not None:
        _need(mask, torch.bool if mask.dtype is torch.bool else torch.uint8, "mask", (T,))
    if grad_in is not None:
        _need(grad_in, torch.float32, "grad_in", (T, E))
    to_bf16 = grad_out is not None and grad_out.dtype is torch.bfloat16
    if grad_out is not None:
        _need(grad_out, torch.bfloat16 if to_bf16 else torch.float32, "grad_out", (T, E))
    if grad_scale is not None:
        _need(grad_scale, torch.float32, "grad_scale", (1,))
    if counts is None:
        counts = _new((M, E), torch.int32, z, stream)
    else:
        _need(counts, torch.int32, "counts", (M, E))
    if loss is None:
        loss = _new((M, 2), torch.float32, z, stream)
    else:
        _need(loss, torch.float32, "loss", (M, 2))
    if prob is not None:
        _need(prob, torch.float32, "prob", (M, E))
    if workspace is None:
        workspace = _new(eqb_balance_loss_workspace_bytes(T, E, M), torch.uint8, z, stream)
    else:
        _need(workspace, torch.uint8, "workspace")
    if err_flag is not None:
        _need(err_flag, torch.int32, "err_flag")
    rc = load().eqb_balance_loss(z.data_ptr(), fp32, topk_idx.data_ptr(), T, E, K, mb_offsets.data_ptr(), M, _p(mask), kind,
                                 alpha, zeta, _p(grad_in), _p(grad_out), to_bf16, _p(grad_scale), counts.data_ptr(),
                                 _p(prob), loss.data_ptr(), workspace.data_ptr(), workspace.numel(), _p(err_flag),
                                 _stream(stream))
    _check(rc, "eqb_balance_loss")
    return loss, counts


def eqb_router_grad_workspace_bytes(T: int, d: int, E: int) -> int:
    return int(load().eqb_router_grad_workspace_bytes(T, d, E))


def eqb_router_grad(dz, x, W_r, dx=None, dW=None, accumulate_dx=False, accumulate_dW=False, workspace=None,
                    err_flag=None, stream=None):
    """Gradients of eqb_router_logits from dz bf16 [T,E]: dx = dz W_r into dx
    bf16 [T,d] and dW = dz^T x into dW fp32 [E,d], each where it is given (or
    added to it, with accumulate_*).  Returns (dx, dW)."""
    T, E = dz.shape
    d = W_r.shape[1]
    _need(dz, torch.bfloat16, "dz")
    _on_current_device(dz, "dz")
    _need(x, torch.bfloat16, "x", (T, d))
    _need(W_r, torch.bfloat16, "W_r", (E, d))
    if dx is not None:
        _need(dx, torch.bfloat16, "dx", (T, d))
    if dW is not None:
        _need(dW, torch.float32, "dW", (E, d))
    if workspace is not None:
        _need(workspace, torch.uint8, "workspace")
    elif dW is not None:
        need = eqb_router_grad_workspace_bytes(T, d, E)
        workspace = _new(need, torch.uint8, dz, stream) if need else None
    if err_flag is not None:
        _need(err_flag, torch.int32, "err_flag")
    rc = load().eqb_router_grad(dz.data_ptr(), x.data_ptr(), W_r.data_ptr(), T, d, E, _p(dx), bool(accumulate_dx), _p(dW),
                                bool(accumulate_dW), _p(workspace), 0 if workspace is None else workspace.numel(),
                                _p(err_flag), _stream(stream))
    _check(rc, "eqb_router_grad")
    return dx, dW


def _dims(t, n, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dim() != n:
        raise ValueError(f"{name} must have {n} dimensions, got {tuple(t.shape)}")
    return t.shape


def _either(t, a, b):
    """The one of two types that t has, else the first, which _need then asks for."""
    return b if isinstance(t, torch.Tensor) and t.dtype is b else a


_GROUP_SCORES = {"max": 0, "top2": 1}


def _one_of(kinds, value, name):
    kind = kinds.get(value)
    if kind is None:
        raise ValueError(f"{name} must be one of {sorted(kinds)}, got {value!r}")
    return kind


def _mask(mask, T):
    if mask is not None:
        _need(mask, _either(mask, torch.bool, torch.uint8), "mask", (T,))


def eqb_gate_topk(z, b, K, score="sigmoid", groups=1, top_groups=1, group_score="max", renorm=True, scale=1.0, mask=None,
                  topk_idx=None, weight=None, err_flag=None, stream=None):
    """The gate: K experts a token by z + b, from the top_groups best of `groups`
    groups of neighbouring experts (group_score "max", or "top2": the sum of a group's two
    largest), and their weights from z: sigmoid or softmax, renormalised over the
    list or not, times scale (see eqb.h).  z bf16 or fp32 [T,E]; b fp32 [E] or
    None; mask bool or uint8 [T].  A closed expert has z or b of -inf.  Returns
    (topk_idx int32 [T,K], -1 where no expert is left, weight fp32 [T,K])."""
    T, E = _dims(z, 2, "z")
    dt = _either(z, torch.bfloat16, torch.float32)
    _need(z, dt, "z")
    _on_current_device(z, "z")
    if b is not None:
        _need(b, torch.float32, "b", (E,))
    kind, two = _one_of(_SCORES, score, "score"), _one_of(_GROUP_SCORES, group_score, "group_score")
    _mask(mask, T)
    if topk_idx is None:
        topk_idx = _new((T, K), torch.int32, z, stream)
    else:
        _need(topk_idx, torch.int32, "topk_idx", (T, K))
    if weight is None:
        weight = _new((T, K), torch.float32, z, stream)
    else:
        _need(weight, torch.float32, "weight", (T, K))
    _need(err_flag, torch.int32, "err_flag")
    rc = load().eqb_gate_topk(z.data_ptr(), dt is torch.float32, _p(b), T, E, K, groups, top_groups, two, kind, bool(renorm),
                              scale, _p(mask), topk_idx.data_ptr(), weight.data_ptr(), _p(err_flag), _stream(stream))
    _check(rc, "eqb_gate_topk")
    return topk_idx, weight


def eqb_gate_grad(z, topk_idx, grad_weight, score="sigmoid", renorm=True, scale=1.0, grad_in=None, grad_out=None, stream=None):
    """Gradient of eqb_gate_topk's weights with respect to z, from grad_weight
    fp32 [T,K]: grad_out (fp32, or bf16 [T,E]; fp32 when not given) = grad_in + d,
    d alone without grad_in; grad_out may be grad_in.  What eqb_balance_loss takes as
    grad_in, and in bf16 eqb_router_grad as dz.  Returns grad_out."""
    T, E = _dims(z, 2, "z")
    K = _dims(topk_idx, 2, "topk_idx")[1]
    dt = _either(z, torch.bfloat16, torch.float32)
    _need(z, dt, "z")
    _on_current_device(z, "z")
    _need(topk_idx, torch.int32, "topk_idx", (T, K))
    if grad_weight is None:
        raise TypeError("grad_weight must be a torch.Tensor")
    _need(grad_weight, torch.float32, "grad_weight", (T, K))
    kind = _one_of(_SCORES, score, "score")
    if grad_in is not None:
        _need(grad_in, torch.float32, "grad_in", (T, E))
    if grad_out is None:
        grad_out = _new((T, E), torch.float32, z, stream)
    to = _either(grad_out, torch.float32, torch.bfloat16)
    _need(grad_out, to, "grad_out", (T, E))
    rc = load().eqb_gate_grad(z.data_ptr(), dt is torch.float32, topk_idx.data_ptr(), grad_weight.data_ptr(), T, E, K, kind,
                              bool(renorm), scale, _p(grad_in), grad_out.data_ptr(), to is torch.bfloat16, _stream(stream))
    _check(rc, "eqb_gate_grad")
    return grad_out


def eqb_expert_rows_workspace_bytes(T: int, K: int, E: int) -> int:
    return int(load().eqb_expert_rows_workspace_bytes(T, K, E))


def eqb_expert_max_blocks(R: int, E: int) -> int:
    """Most blocks of 128 rows that R rows of E experts can have."""
    return int(load().eqb_expert_max_blocks(R, E))


def eqb_expert_rows(topk_idx, E, offsets=None, blocks=None, slot=None, entry=None, workspace=None, stream=None):
    """The experts' rows from the lists topk_idx int32 [T,K]: the entries sorted by
    expert, in ascending order within one.  Returns (offsets int32 [E+1],
    blocks int32 [E+1], slot int32 [T,K], entry int32 [T*K]); see eqb.h."""
    T, K = _dims(topk_idx, 2, "topk_idx")
    _need(topk_idx, torch.int32, "topk_idx")
    _on_current_device(topk_idx, "topk_idx")
    made = []
    for t, name, shape in ((offsets, "offsets", (E + 1,)), (blocks, "blocks", (E + 1,)), (slot, "slot", (T, K)),
                           (entry, "entry", (T * K,))):
        if t is None:
            t = _new(shape, torch.int32, topk_idx, stream)
        else:
            _need(t, torch.int32, name, shape)
        made.append(t)
    offsets, blocks, slot, entry = made
    if workspace is None:
        need = eqb_expert_rows_workspace_bytes(T, K, E)
        workspace = _new(need, torch.uint8, topk_idx, stream) if need else None
    else:
        _need(workspace, torch.uint8, "workspace")
    rc = load().eqb_expert_rows(topk_idx.data_ptr(), T, K, E, offsets.data_ptr(), blocks.data_ptr(), slot.data_ptr(),
                                entry.data_ptr(), _p(workspace), 0 if workspace is None else workspace.numel(), _stream(stream))
    _check(rc, "eqb_expert_rows")
    return offsets, blocks, slot, entry


_E4M3 = torch.float8_e4m3fn


def _up(n):
    return (n + 127) // 128


def eqb_quant_rows(x, slot=None, q=None, scale=None, err_flag=None, stream=None):
    """x bf16 [T,d] in 8 bits, with a scale for every 128 neighbours of a row.
    With slot int32 [T,K] (eqb_expert_rows) row t goes to the rows slot[t] of q
    [T*K,d], those of -1 left out.  Without, every row of x is read: sorted rows
    behind the last expert's have to hold something finite, or be left out by a slot
    [R,1] (see eqb.h).  Returns (q float8_e4m3fn, scale fp32 [rows, ceil(d/128)])."""
    T, d = _dims(x, 2, "x")
    _need(x, torch.bfloat16, "x")
    _on_current_device(x, "x")
    K, R = 1, T
    if slot is not None:
        K = _dims(slot, 2, "slot")[1]
        _need(slot, torch.int32, "slot", (T, K))
        R = T * K
    if q is None:
        q = _new((R, d), _E4M3, x, stream)
    else:
        _need(q, _E4M3, "q", (R, d))
    if scale is None:
        scale = _new((R, _up(d)), torch.float32, x, stream)
    else:
        _need(scale, torch.float32, "scale", (R, _up(d)))
    _need(err_flag, torch.int32, "err_flag")
    rc = load().eqb_quant_rows(x.data_ptr(), T, d, _p(slot), K, q.data_ptr(), scale.data_ptr(), _p(err_flag), _stream(stream))
    _check(rc, "eqb_quant_rows")
    return q, scale


def eqb_quant_cols(x, offsets, blocks, entry=None, K=None, q=None, scale=None, err_flag=None, stream=None):
    """The experts' rows in 8 bits, turned, with a scale for every 128 rows of an
    expert and column: the operands of eqb_expert_wgrad.  x bf16 [R,c] in sorted
    rows, or with entry int32 [R] (eqb_expert_rows) and K, the length of the lists,
    [T,c] by token: entry i is of token i // K.  Returns (q float8_e4m3fn [c, 128 P],
    scale fp32 [P,c]), P = eqb_expert_max_blocks(R, E) unless q says otherwise."""
    if K is None:
        if entry is not None:
            raise ValueError("entry needs K: the lists' length says which token an entry is of")
        K = 1
    T, c = _dims(x, 2, "x")
    _need(x, torch.bfloat16, "x")
    _on_current_device(x, "x")
    E = _dims(offsets, 1, "offsets")[0] - 1
    _need(offsets, torch.int32, "offsets")
    if blocks is None:
        raise TypeError("blocks must be a torch.Tensor")
    _need(blocks, torch.int32, "blocks", (E + 1,))
    R = T
    if entry is not None:
        R = _dims(entry, 1, "entry")[0]
        _need(entry, torch.int32, "entry")
    if q is None:
        P = eqb_expert_max_blocks(R, E) if scale is None else _dims(scale, 2, "scale")[0]
        q = _new((c, max(P, 0) * 128), _E4M3, x, stream)
    else:
        P = _dims(q, 2, "q")[1] // 128
        _need(q, _E4M3, "q", (c, P * 128))
    if scale is None:
        scale = _new((max(P, 0), c), torch.float32, x, stream)
    else:
        _need(scale, torch.float32, "scale", (P, c))
    _need(err_flag, torch.int32, "err_flag")
    rc = load().eqb_quant_cols(x.data_ptr(), T, c, _p(entry), R, K, offsets.data_ptr(), blocks.data_ptr(), E, P, q.data_ptr(),
                               scale.data_ptr(), _p(err_flag), _stream(stream))
    _check(rc, "eqb_quant_cols")
    return q, scale


def eqb_quant_blocks(w, q=None, scale=None, q_t=None, scale_t=None, turned=False, err_flag=None, stream=None):
    """Matrices w bf16 or fp32 [E,n,d] in 8 bits with a scale for every 128 x 128,
    and with turned (or where q_t and scale_t are given) their transposes too.
    Returns (q, scale), or (q, scale, q_t, scale_t)."""
    E, n, d = _dims(w, 3, "w")
    dt = _either(w, torch.bfloat16, torch.float32)
    _need(w, dt, "w")
    _on_current_device(w, "w")
    turned = turned or q_t is not None or scale_t is not None
    made = []
    for t, name, dtype, shape, want in ((q, "q", _E4M3, (E, n, d), True), (scale, "scale", torch.float32, (E, _up(n), _up(d)), True),
                                        (q_t, "q_t", _E4M3, (E, d, n), turned),
                                        (scale_t, "scale_t", torch.float32, (E, _up(d), _up(n)), turned)):
        if t is not None:
            _need(t, dtype, name, shape)
        elif want:
            t = _new(shape, dtype, w, stream)
        made.append(t)
    q, scale, q_t, scale_t = made
    _need(err_flag, torch.int32, "err_flag")
    rc = load().eqb_quant_blocks(w.data_ptr(), dt is torch.float32, E, n, d, q.data_ptr(), scale.data_ptr(), _p(q_t), _p(scale_t),
                                 _p(err_flag), _stream(stream))
    _check(rc, "eqb_quant_blocks")
    return (q, scale, q_t, scale_t) if turned else (q, scale)


def eqb_expert_matmul(q, scale, w, w_scale, offsets, out=None, err_flag=None, stream=None):
    """Every expert's rows times its weights in 8 bits: out[r] = q_r w_e^T for the
    rows offsets[e] .. offsets[e+1]-1.  q [R,d] and scale [R, ceil(d/128)] from
    eqb_quant_rows, w [E,n,d] and w_scale from eqb_quant_blocks (the transposed pair
    for the gradient of the input), offsets int32 [E+1] from eqb_expert_rows.
    out: bf16 (when not given) or fp32 [R,n]; rows behind the last expert's are
    left as they are.  Returns out."""
    R, d = _dims(q, 2, "q")
    E, n, _ = _dims(w, 3, "w")
    _need(q, _E4M3, "q")
    _on_current_device(q, "q")
    _need(w, _E4M3, "w", (E, n, d))
    for t, name, shape in ((scale, "scale", (R, _up(d))), (w_scale, "w_scale", (E, _up(n), _up(d)))):
        if t is None:
            raise TypeError(f"{name} must be a torch.Tensor")
        _need(t, torch.float32, name, shape)
    if offsets is None:
        raise TypeError("offsets must be a torch.Tensor")
    _need(offsets, torch.int32, "offsets", (E + 1,))
    if out is None:
        out = _new((R, n), torch.bfloat16, q, stream)
    to = _either(out, torch.bfloat16, torch.float32)
    _need(out, to, "out", (R, n))
    _need(err_flag, torch.int32, "err_flag")
    rc = load().eqb_expert_matmul(q.data_ptr(), scale.data_ptr(), w.data_ptr(), w_scale.data_ptr(), offsets.data_ptr(), R, n, d, E,
                                  out.data_ptr(), to is torch.float32, _p(err_flag), _stream(stream))
    _check(rc, "eqb_expert_matmul")
    return out


def eqb_expert_wgrad(a, a_scale, b, b_scale, blocks, dW=None, accumulate=False, err_flag=None, stream=None):
    """The gradient of eqb_expert_matmul's weights in 8 bits: dW[e] = a_e b_e^T over
    the expert's rows, a [n, 128 P] and b [d, 128 P] from eqb_quant_cols over the
    same rows (of the output's gradient and of the input), blocks int32 [E+1] from
    eqb_expert_rows.  dW fp32 [E,n,d], with accumulate added to.  Returns dW."""
    n, p = _dims(a, 2, "a")
    d = _dims(b, 2, "b")[0]
    P = p // 128
    E = _dims(blocks, 1, "blocks")[0] - 1
    _need(a, _E4M3, "a", (n, P * 128))
    _on_current_device(a, "a")
    _need(b, _E4M3, "b", (d, P * 128))
    for t, name, shape in ((a_scale, "a_scale", (P, n)), (b_scale, "b_scale", (P, d))):
        if t is None:
            raise TypeError(f"{name} must be a torch.Tensor")
        _need(t, torch.float32, name, shape)
    _need(blocks, torch.int32, "blocks")
    if dW is None:
        if accumulate:
            raise ValueError("accumulate needs dW")
        dW = _new((E, n, d), torch.float32, a, stream)
    else:
        _need(dW, torch.float32, "dW", (E, n, d))
    _need(err_flag, torch.int32, "err_flag")
    rc = load().eqb_expert_wgrad(a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(), blocks.data_ptr(), P, n, d, E,
                                 dW.data_ptr(), bool(accumulate), _p(err_flag), _stream(stream))
    _check(rc, "eqb_expert_wgrad")
    return dW


def eqb_expert_combine(rows, slot, weight=None, out=None, stream=None):
    """out[t] = sum_k weight[t,k] rows[slot[t,k]] (bf16 [T,n]) over the slots that are
    rows, 1 for every weight when not given.  rows bf16 [R,n]; slot int32 [T,K];
    weight fp32 [T,K].  Returns out."""
    R, n = _dims(rows, 2, "rows")
    T, K = _dims(slot, 2, "slot")
    _need(rows, torch.bfloat16, "rows")
    _on_current_device(rows, "rows")
    _need(slot, torch.int32, "slot")
    if weight is not None:
        _need(weight, torch.float32, "weight", (T, K))
    if out is None:
        out = _new((T, n), torch.bfloat16, rows, stream)
    else:
        _need(out, torch.bfloat16, "out", (T, n))
    rc = load().eqb_expert_combine(rows.data_ptr(), slot.data_ptr(), _p(weight), T, R, n, K, out.data_ptr(), _stream(stream))
    _check(rc, "eqb_expert_combine")
    return out


def eqb_expert_combine_grad(grad, rows, slot, weight=None, grad_rows=None, grad_weight=None, stream=None):
    """Gradients of eqb_expert_combine from grad bf16 [T,n]: grad_rows (bf16 [R,n],
    rows without a slot left as they are; may be rows itself) and grad_weight
    (fp32 [T,K]), each where it is given.  Returns (grad_rows, grad_weight)."""
    T, n = _dims(grad, 2, "grad")
    R = _dims(rows, 2, "rows")[0]
    K = _dims(slot, 2, "slot")[1]
    _need(grad, torch.bfloat16, "grad")
    _on_current_device(grad, "grad")
    _need(rows, torch.bfloat16, "rows", (R, n))
    _need(slot, torch.int32, "slot", (T, K))
    if weight is not None:
        _need(weight, torch.float32, "weight", (T, K))
    if grad_rows is not None:
        _need(grad_rows, torch.bfloat16, "grad_rows", (R, n))
    if grad_weight is not None:
        _need(grad_weight, torch.float32, "grad_weight", (T, K))
    rc = load().eqb_expert_combine_grad(grad.data_ptr(), rows.data_ptr(), slot.data_ptr(), _p(weight), T, R, n, K, _p(grad_rows),
                                        _p(grad_weight), _stream(stream))
    _check(rc, "eqb_expert_combine_grad")
    return grad_rows, grad_weight


_data_ptr, _numel = torch.Tensor.data_ptr, torch.Tensor.numel
_get_device, _is_contiguous = torch.Tensor.get_device, torch.Tensor.is_contiguous
_GRAD_TYPES = {torch.float32, torch.bfloat16}


class EqbAdamW:
    """AdamW over a list of tensors, one launch for up to 400 of them (see
    eqb_adamw_step in eqb.h).

    params  fp32 or bf16 tensors, contiguous, on one GPU
    state_bits  32: exp_avg, exp_avg_sq fp32.  8: exp_avg (m) and exp_avg_sq
            (the root of the second moment) torch.float8_e4m3fn, with an fp32
            scale for every 256 elements in avg_scale and sq_scale; for
            beta2 up to 0.95 (eqb.h says what becomes of larger ones).
    exp_avg, exp_avg_sq, avg_scale, sq_scale  lists of tensors to keep the
            states in (continued from a checkpoint, say); zeros when not given,
            written on the stream that is current when the object is made
    copies  bf16 tensors (or None) that receive the new value of the fp32
            parameter beside them, rounded, e.g. the W_r that the projection
            reads

    The object holds the tensors.  A parameter that has moved to another
    storage is refused by step(); states and copies that are moved away from
    their storage are not followed."""

    BLOCK = 256

    def __init__(self, params, state_bits=32, exp_avg=None, exp_avg_sq=None, avg_scale=None, sq_scale=None, copies=None):
        self.params = list(params)
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.state_bits = state_bits
        kind = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        for i, p in enumerate(self.params):
            if not isinstance(p, torch.Tensor):
                raise TypeError(f"params[{i}] must be a torch.Tensor")
            if p.dtype not in _GRAD_TYPES:
                raise TypeError(f"params[{i}] must be torch.float32 or torch.bfloat16, got {p.dtype}")
            if not (p.is_cuda and p.is_contiguous()):
                _need(p, p.dtype, f"params[{i}]")

        def own(given, name, shapes, dtype):
            if given is None:
                return [torch.zeros(s, dtype=dtype, device=p.device) for p, s in zip(self.params, shapes)]
            given = list(given)
            if len(given) != len(self.params):
                raise ValueError(f"{name} must have {len(self.params)} tensors, got {len(given)}")
            for i, (t, s) in enumerate(zip(given, shapes)):
                if t is None:
                    raise TypeError(f"{name}[{i}] must be a torch.Tensor")
                if not (type(t) is torch.Tensor and t.dtype is dtype and t.is_cuda and t.shape == s and t.is_contiguous()):
                    _need(t, dtype, f"{name}[{i}]", s)
            return given

        shapes = [p.shape for p in self.params]
        self.exp_avg = own(exp_avg, "exp_avg", shapes, kind)
        self.exp_avg_sq = own(exp_avg_sq, "exp_avg_sq", shapes, kind)
        self.avg_scale = self.sq_scale = None
        if state_bits == 8:
            blocks = [((p.numel() + self.BLOCK - 1) // self.BLOCK,) for p in self.params]
            self.avg_scale = own(avg_scale, "avg_scale", blocks, torch.float32)
            self.sq_scale = own(sq_scale, "sq_scale", blocks, torch.float32)
        elif avg_scale is not None or sq_scale is not None:
            raise ValueError("avg_scale and sq_scale belong to state_bits=8")
        self.copies = [None] * len(self.params) if copies is None else list(copies)
        if len(self.copies) != len(self.params):
            raise ValueError(f"copies must have {len(self.params)} entries, got {len(self.copies)}")
        for i, (c, p) in enumerate(zip(self.copies, self.params)):
            if c is not None and p.dtype is not torch.float32:
                raise TypeError(f"copies[{i}] is given but params[{i}] is not torch.float32")
            _need(c, torch.bfloat16, f"copies[{i}]", p.shape)
        states = self.exp_avg + self.exp_avg_sq + (self.avg_scale or []) + (self.sq_scale or []) + [
            c for c in self.copies if c is not None]
        if len({t.device for t in self.params + states}) > 1:
            raise ValueError("all tensors must be on one device")
        # aliases: what the table points to stays allocated whatever becomes of the tensors above
        self._held = [t.detach() for t in self.params + states]
        # one tensor for every version counter: views share their base's
        base = [t if t._base is None else t._base for t in self.params + self.copies if t is not None]
        self._written = list({id(t): t for t in base}.values())
        self._ptrs = [p.data_ptr() for p in self.params]
        self._numels = [p.numel() for p in self.params]
        self._device = [p.get_device() for p in self.params]
        self._dtypes = None  # of the last step's gradients: the table's grad_bf16
        self._whole = [True] * len(self.params)
        self._table = (AdamwTensor * len(self.params))()
        # the grad field of every entry, as one strided row
        words = ctypes.sizeof(AdamwTensor) // 8
        self._grad_words = memoryview(self._table).cast("B").cast("Q")[AdamwTensor.grad.offset // 8::words]
        for i, (e, p) in enumerate(zip(self._table, self.params)):
            e.param, e.n, e.param_bf16 = p.data_ptr(), p.numel(), p.dtype is torch.bfloat16
            e.exp_avg, e.exp_avg_sq = self.exp_avg[i].data_ptr(), self.exp_avg_sq[i].data_ptr()
            if state_bits == 8:
                e.avg_scale, e.sq_scale = self.avg_scale[i].data_ptr(), self.sq_scale[i].data_ptr()
            e.copy = _p(self.copies[i])

    def _point_to(self, grads):
        """The gradients' addresses into the table, after their checks; whether none is missing."""
        try:  # the checks of all of them at once: hundreds of tensors take longer one by one than their step
            ptrs = list(map(_data_ptr, grads))
            dtypes = [g.dtype for g in grads]
            fits = (list(map(_get_device, grads)) == self._device and list(map(_is_contiguous, grads)) == self._whole and
                    list(map(_numel, grads)) == self._numels and (dtypes == self._dtypes or _GRAD_TYPES.issuperset(dtypes)))
        except (TypeError, AttributeError):
            fits = False
        if not fits:  # a gradient is missing, or one that is refused
            ptrs, dtypes = [], []
            for i, (g, p) in enumerate(zip(grads, self.params)):
                if g is not None:
                    _need(g, g.dtype if getattr(g, "dtype", None) in _GRAD_TYPES else torch.float32, f"grads[{i}]")
                    if g.numel() != p.numel():
                        raise ValueError(f"grads[{i}] must have shape {tuple(p.shape)} or as many elements, got {tuple(g.shape)}")
                    if g.device != p.device:
                        raise ValueError(f"grads[{i}] is on {g.device}, its parameter on {p.device}")
                ptrs.append(0 if g is None else g.data_ptr())
                dtypes.append(torch.float32 if g is None else g.dtype)
        if dtypes != self._dtypes:
            for e, t in zip(self._table, dtypes):
                e.grad_bf16 = t is torch.bfloat16
            self._dtypes = dtypes
        self._grad_words[:] = memoryview(array("Q", ptrs))
        return fits

    def step(self, grads, lr, step, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, grad_scale=None, err_flag=None,
             stream=None):
        """One step (step = 1 for the first) with `grads`, a list of fp32 or
        bf16 tensors of the parameters' shapes (or flat); a parameter whose
        entry is None is left as it is.  grad_scale: fp32 CUDA tensor [1] that every
        gradient is multiplied by."""
        if len(grads) != len(self.params):
            raise ValueError(f"grads must have {len(self.params)} entries, got {len(grads)}")
        if list(map(_data_ptr, self.params)) != self._ptrs:
            raise ValueError("a parameter has moved to another storage: make a new EqbAdamW")
        if self.params:
            _on_current_device(self.params[0], "params[0]")
        all_given = self._point_to(grads)
        _need(grad_scale, torch.float32, "grad_scale", (1,))
        _need(err_flag, torch.int32, "err_flag")
        rc = load().eqb_adamw_step(self._table, len(self.params), self.state_bits, float(lr), int(step), float(beta1),
                                   float(beta2), float(eps), float(weight_decay), _p(grad_scale), _p(err_flag),
                                   _stream(stream))
        # autograd has to know that values it may have saved are gone
        increment_version(self._written if all_given else [
            t for p, c, g in zip(self.params, self.copies, grads) if g is not None for t in (p, c) if t is not None])
        _check(rc, "eqb_adamw_step")
