"""The chain from score gradients to the router's gradients: dL/ds of the experts'
path, LEI added to it, through the sigmoid, the balance loss added, and the
projection's gradients (examples/router_training.py), against autograd in 64 bits."""
import os
import sys

import pytest
import torch

import paper_2609_28053_gb300 as eqb

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("alpha,zeta,eta", [(0.02, 1e-4, 0.05), (0.0, 0.0, 0.05), (0.02, 0.0, 0.0)])
def test_joined_gradients_against_autograd(alpha, zeta, eta):
    """dz is rounded to bf16 (2^-8 of itself; before that 2e-5 of its terms), so dW
    and dx are off by that of the magnitudes of their products."""
    from router_training import RouterTrainer, tokens

    t = RouterTrainer(512, 128, 16, 2, 2, accumulate=2, alpha=alpha, zeta=zeta, eta=eta, c=1.0)
    W = t.W_r.double()
    xs = [tokens(t.T, t.d, 5), tokens(t.T, t.d, 6)]
    g = torch.Generator(device="cuda").manual_seed(3)
    grad_s = [0.1 * torch.randn(t.T, t.E, generator=g, device="cuda") for _ in xs]
    off = t.offsets.tolist()
    dW, sizeW = torch.zeros(t.E, t.d, dtype=torch.float64, device="cuda"), torch.zeros(t.E, t.d, dtype=torch.float64, device="cuda")
    for x, gs in zip(xs, grad_s):
        zb = eqb.eqb_router_logits(x, t.W_r)
        idx = eqb.eqb_route_topk(zb, t.bias, t.K, topk_idx=torch.empty(t.T, t.K, dtype=torch.int32, device="cuda"))[0].long()
        z = zb.double().requires_grad_()
        s = torch.sigmoid(z)
        loss = (gs.double() * s).sum()  # the experts' path, to first order in s
        for a, b in zip(off, off[1:]):
            n = b - a
            f = torch.bincount(idx[a:b].flatten(), minlength=t.E).double()
            rho = f * t.E / (t.K * n) - 1
            xi = rho.abs().max() / t.c
            loss = loss + (t.eta * torch.tanh(xi) / xi * rho * s[a:b]).sum()
            part = t.alpha * (f / (t.K * n) * torch.softmax(z[a:b], 1).mean(0)).sum()
            part = part + t.zeta * torch.logsumexp(z[a:b], 1).square().mean()
            loss = loss + part / (t.accumulate * t.M)
        (dz,) = torch.autograd.grad(loss, [z])
        dW += dz.t() @ x.double()
        sizeW += dz.abs().t() @ x.double().abs()
    t.step(xs, grad_s)
    assert t.err.item() == 0
    assert torch.all((t.dW.double() - dW).abs() <= (2.0 ** -8 + 1e-4) * sizeW)
    dx, size = dz @ W, dz.abs() @ W.abs()  # of the last batch
    assert torch.all((t.dx.double() - dx).abs() <= (2.0 ** -8 + 1e-4) * size + 2.0 ** -8 * dx.abs())
