"""eqb_gate_topk's results at the ends of fp32: factors near its largest value.
Tolerances are those of the gate's other tests."""
import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("T", [64, 9000])
@pytest.mark.parametrize("level", [-3.0, 0.0, 3.0])
@pytest.mark.parametrize("K", [1, 4])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_a_factor_near_the_largest(T, level, K, score):
    """The weights sum up to it, so none passes it."""
    g = torch.Generator().manual_seed(T)
    z = torch.randn(T, 64, generator=g) + level
    scale = 3.4e38
    idx, w = eqb.eqb_gate_topk(z.cuda(), None, K, score=score, scale=scale)
    want = ref.choose(z, None, K)
    assert torch.equal(idx.cpu(), want)
    exact = ref.shares(z, want, score, True, scale)
    spread = float(z.max() - z.min()) + float(z.abs().max())
    assert torch.all((w.cpu().double() - exact).abs() <= (102 + 2 * spread) * U * exact)
