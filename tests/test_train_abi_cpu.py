"""Host-side refusals of the training entry points: nothing is launched, so no GPU is needed."""
import ctypes

import pytest

import paper_2609_28053_gb300 as eqb
from paper_2609_28053_gb300 import _lib

INVALID, UNSUPPORTED = 1, 2
FAKE = ctypes.c_void_p(0x10000)
OFF4 = ctypes.c_void_p(0x10004)
NULL = None


@pytest.fixture(scope="module")
def lib():
    return eqb.load()


def test_balance_loss_refuses(lib):
    ws = lib.eqb_balance_loss_workspace_bytes(100, 64, 2)
    assert ws > 0 and lib.eqb_balance_loss_workspace_bytes(100, 64, 0) == 0

    def call(z=FAKE, idx=FAKE, T=100, E=64, K=4, off=FAKE, M=2, mask=NULL, score=0, alpha=0.1, zeta=0.0, gi=NULL, go=FAKE,
             bf16=0, gs=NULL, counts=FAKE, prob=NULL, loss=FAKE, w=FAKE, wb=ws):
        return lib.eqb_balance_loss(z, 0, idx, T, E, K, off, M, mask, score, alpha, zeta, gi, go, bf16, gs, counts, prob, loss,
                                    w, wb, NULL, NULL)

    assert call(E=60) == UNSUPPORTED
    assert call(E=1032) == UNSUPPORTED
    assert call(K=0) == INVALID and call(K=64) == INVALID and call(K=32) == UNSUPPORTED
    assert call(T=-1) == INVALID and call(T=2 ** 31) == UNSUPPORTED
    assert call(M=0) == INVALID and call(M=2 ** 20 + 1) == UNSUPPORTED
    assert call(score=2) == INVALID
    assert call(score=1, zeta=0.1) == INVALID
    assert call(alpha=float("nan")) == INVALID and call(zeta=float("inf")) == INVALID
    for name in ("z", "idx", "off", "counts"):
        assert call(**{name: NULL}) == INVALID
    assert call(w=NULL) == INVALID and call(wb=ws - 1) == INVALID and call(w=OFF4) == INVALID
    assert call(z=OFF4) == INVALID and call(go=OFF4) == INVALID and call(gi=OFF4) == INVALID
    assert call(gi=FAKE, go=NULL) == INVALID
    assert call(gi=FAKE, go=FAKE, bf16=1) == INVALID  # fp32 in, bf16 out, one buffer


def test_router_grad_refuses(lib):
    ws = lib.eqb_router_grad_workspace_bytes(65536, 4096, 128)
    assert ws > 0
    assert lib.eqb_router_grad_workspace_bytes(65536, 4090, 128) == 0

    def call(dz=FAKE, x=FAKE, W=FAKE, T=65536, d=4096, E=128, dx=FAKE, dW=FAKE, w=FAKE, wb=ws):
        return lib.eqb_router_grad(dz, x, W, T, d, E, dx, 0, dW, 0, w, wb, NULL, NULL)

    assert call(d=4090) == UNSUPPORTED and call(E=24) == UNSUPPORTED and call(E=272) == UNSUPPORTED
    assert call(T=-1) == INVALID and call(d=0) == INVALID and call(T=2 ** 31) == UNSUPPORTED
    assert call(dz=NULL) == INVALID and call(x=NULL) == INVALID and call(W=NULL) == INVALID
    assert call(dx=OFF4) == INVALID and call(dW=OFF4) == INVALID and call(dz=OFF4) == INVALID
    assert call(w=NULL) == INVALID and call(wb=ws - 1) == INVALID and call(w=OFF4) == INVALID
    assert call(dx=NULL, dW=NULL) == 0  # nothing asked for


def test_adamw_refuses(lib):
    def call(bits=32, lr=1e-3, step=1, b1=0.9, b2=0.95, eps=1e-8, wd=0.1, count=1, **kw):
        t = (_lib.AdamwTensor * 1)()
        e = t[0]
        e.param = e.grad = e.exp_avg = e.exp_avg_sq = e.avg_scale = e.sq_scale = 0x10000
        e.n = 10
        for k, v in kw.items():
            setattr(e, k, v)
        return lib.eqb_adamw_step(t, count, bits, lr, step, b1, b2, eps, wd, NULL, NULL, NULL)

    assert call(bits=16) == INVALID
    assert call(count=-1) == INVALID
    assert lib.eqb_adamw_step(NULL, 1, 32, 1e-3, 1, 0.9, 0.95, 1e-8, 0.1, NULL, NULL, NULL) == INVALID
    for kw in (dict(lr=-1.0), dict(lr=float("nan")), dict(step=0), dict(b1=1.0), dict(b2=-0.1), dict(b2=float("nan")), dict(eps=0.0),
               dict(wd=-1.0), dict(n=-1), dict(n=2 ** 41), dict(param=None), dict(exp_avg=None), dict(exp_avg_sq=None),
               dict(param=0x10001), dict(grad=0x10002), dict(exp_avg=0x10001)):
        assert call(**kw) == INVALID, kw
    assert call(bits=8, avg_scale=None) == INVALID and call(bits=8, sq_scale=0x10002) == INVALID
    assert call(copy=0x10000, param_bf16=1) == INVALID
    # nothing to do
    assert call(count=0) == 0 and call(n=0, param=None) == 0 and call(grad=None) == 0


def test_bindings_refuse_host_tensors():
    import torch
    z = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        eqb.eqb_balance_loss(z, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int64), 0.1)
    with pytest.raises(ValueError, match="CUDA"):
        eqb.eqb_router_grad(z, z, z)
    with pytest.raises(ValueError, match="CUDA"):
        eqb.EqbAdamW([torch.zeros(4)])
    with pytest.raises(TypeError):
        eqb.EqbAdamW([torch.zeros(4, dtype=torch.float16)])
