"""The links of a layer's backward pass, each against 64 bits from what the call before it
has stored, so that a bound is one call's rounding and not the 8 bits' of all: from the
rows to the gate weights' gradient, from there to the logits', and through the balance
loss to the router's.

A dot product of n products: a lane adds 8 ceil(n / 256) of them, one rounding each, and
five additions join the lanes: (8 ceil(n / 256) + 5) 2^-24 of the sum of magnitudes.  A
gradient of the gate: the bound of the gate's own tests.  Each test shows that zeros and
the other sign would not pass."""
import numpy as np
import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb
import train_reference

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def layer(T, d, n, E, K, groups, score, seed, mask=None):
    """Forward and backward; everything that the calls have stored."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    W = torch.randn(E, n, d, generator=g, device="cuda") * d ** -0.5
    z = torch.randn(T, E, generator=g, device="cuda").bfloat16()
    b = torch.randn(E, generator=g, device="cuda") * 0.2
    dy = torch.randn(T, n, generator=g, device="cuda").bfloat16()
    gate = {"score": score, "renorm": True, "scale": 2.5}
    idx, w = eqb.eqb_gate_topk(z, b, K, groups=groups, top_groups=max(1, groups // 2), mask=mask, **gate)
    offsets, blocks, slot, entry = eqb.eqb_expert_rows(idx, E)
    rows = eqb.eqb_expert_matmul(*eqb.eqb_quant_rows(x, slot), *eqb.eqb_quant_blocks(W), offsets)
    g, dw = eqb.eqb_expert_combine_grad(dy, rows, slot, w, grad_rows=torch.zeros_like(rows), grad_weight=torch.empty_like(w))
    dz = eqb.eqb_gate_grad(z, idx, dw, **gate)
    return {"z": z, "dy": dy, "idx": idx, "w": w, "slot": slot, "rows": rows, "g": g, "dw": dw, "dz": dz, "gate": gate}


def holds(got, want, tol):
    """Within the bound, which most values' zero and other sign are not."""
    got, want = got.double().cpu(), want.cpu()
    tol = tol.cpu()
    assert torch.all((got - want).abs() <= tol)
    told = want.abs() > tol  # zero would not pass, nor would -want, which is twice as far
    there = want != 0
    assert told[there].double().mean() > 0.9


SHAPES = [(300, 256, 192, 16, 2, 1, "sigmoid"), (700, 400, 144, 32, 4, 4, "softmax"), (9, 128, 1040, 64, 8, 8, "sigmoid"),
          (5000, 144, 272, 8, 7, 1, "softmax")]


@pytest.mark.parametrize("T,d,n,E,K,groups,score", SHAPES)
@pytest.mark.parametrize("padded", [False, True])
def test_rows_to_weights_to_logits(T, d, n, E, K, groups, score, padded):
    mask = torch.arange(T, device="cuda") % 3 != 0 if padded else None
    s = layer(T, d, n, E, K, groups, score, T, mask)
    here = s["slot"] >= 0
    at = s["slot"].long().clamp(min=0)
    terms = s["dy"].double()[:, None] * s["rows"].double()[at]
    dw = torch.where(here, terms.sum(2), 0.0)
    tol = (8 * -(-n // 256) + 5) * U * 1.001 * terms.abs().sum(2)
    holds(s["dw"], dw, tol)
    # the rows' gradients: one product, rounded to fp32 and to bf16
    rows = s["w"].double()[:, :, None] * s["dy"].double()[:, None]
    holds(s["g"].double()[at][here], rows[here], (2.0 ** -8 + 2.0 ** -23) * rows[here].abs())
    z, idx = s["z"].cpu(), s["idx"].cpu()
    dz, size = ref.gate_grad(z, idx, s["dw"].cpu(), **s["gate"])
    spread = float(z.double().max() - z.double().min()) + float(z.double().abs().max())
    holds(s["dz"], dz, (102 + 2 * spread + 4 * K) * U * size)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_on_into_the_balance_loss(score):
    """dL/dz with the balance loss's gradient in it, by the documented formula, rounded to bf16."""
    T, d, n, E, K = 256, 128, 64, 16, 2
    s = layer(T, d, n, E, K, 1, "sigmoid", 6)
    off = torch.tensor([0, 100, T], device="cuda")
    both = torch.empty(T, E, dtype=torch.bfloat16, device="cuda")
    alpha = 1e4
    eqb.eqb_balance_loss(s["z"], s["idx"], off, alpha, score=score, grad_in=s["dz"], grad_out=both)
    _, _, _, grad, size = train_reference.balance(s["z"].double().cpu().numpy(), s["idx"].cpu().numpy(), [0, 100, T], score, alpha, 0.0)
    want = s["dz"].double().cpu() + torch.from_numpy(grad)
    # its terms within the 2e-5 of the balance loss's own tests, an addition to dz, and the rounding to bf16
    tol = 2e-5 * torch.from_numpy(size) + U * want.abs()
    holds(both, want, tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs())
    # without the balance loss, and with it taken off, it would not pass
    for other in (s["dz"].double().cpu(), s["dz"].double().cpu() - torch.from_numpy(grad)):
        far = (other - want).abs() > tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
        assert far[torch.from_numpy(np.abs(grad) > 0.1)].double().mean() > 0.9
