"""The router's training step as a whole: projection, routing, balance loss,
projection gradients and AdamW together (examples/router_training.py)."""
import os
import sys

import pytest
import torch

import paper_2609_28053_gb300 as eqb

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_the_loss_balances_the_router(bits):
    """MaxVio of a router that the tokens' common component has made uneven
    falls below a third of what it was, and the loss toward alpha / E."""
    from router_training import RouterTrainer, tokens

    t = RouterTrainer(4096, 256, 16, 2, 2, state_bits=bits)
    first = None
    for s in range(80):
        loss, vio = t.step([tokens(t.T, t.d, 100 + 2 * s + i) for i in range(t.accumulate)])
        if first is None:
            first = (loss.item(), vio[0].item())
    assert t.err.item() == 0
    assert first[1] > 1.0
    assert vio[0].item() < first[1] / 3
    assert t.alpha / t.E * 0.99 < loss.item() < first[0]
    assert torch.equal(t.W_r, t.master.bfloat16())


def test_one_step_against_64_bits():
    """The weight's gradient of one step from the formulas: dz in bf16 (2^-8 of
    itself), summed over T tokens whose signs are mixed."""
    from router_training import RouterTrainer, tokens

    t = RouterTrainer(512, 128, 16, 2, 2, accumulate=2)
    W = t.W_r.double()
    xs = [tokens(t.T, t.d, 5), tokens(t.T, t.d, 6)]
    want = torch.zeros(t.E, t.d, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    off = t.offsets.tolist()
    for x in xs:
        z = eqb.eqb_router_logits(x, t.W_r).double()
        idx = torch.topk(z, t.K).indices
        for a, b in zip(off, off[1:]):
            n = b - a
            F = torch.bincount(idx[a:b].flatten(), minlength=t.E).double() / (t.K * n)
            p = torch.softmax(z[a:b], 1)
            lse = torch.logsumexp(z[a:b], 1, keepdim=True)
            d = (t.alpha / n * p * (F - (p @ F)[:, None]) + 2 * t.zeta / n * lse * p) / (t.accumulate * t.M)
            want += d.t() @ x[a:b].double()
            size += d.abs().t() @ x[a:b].double().abs()
    t.step(xs)
    # a tie in the bf16 logits may be broken otherwise by topk above: it moves F by 1 / (K n)
    assert torch.all((t.dW.double() - want).abs() <= (2.0 ** -8 + 1e-3) * size)
