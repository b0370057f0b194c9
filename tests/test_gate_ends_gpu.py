"""eqb_gate_topk's and eqb_gate_grad's results at the ends of fp32: factors near its
largest value, and sigmoids near and below its least normal one.  Tolerances are those
of the gate's other tests; a result below 2^-126 is off by a few steps of 2^-149, of
which the factor makes as many more as it is large."""
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


@pytest.mark.parametrize("T", [64, 9000])
@pytest.mark.parametrize("fp32", [False, True])
def test_sigmoids_below_the_least_normal_number(T, fp32):
    """sigma(z) is exp(z) from -17 down, and a number of fp32 until -103."""
    z = torch.linspace(-110.0, -80.0, T * 64).view(T, 64)
    z = z if fp32 else z.bfloat16()
    idx, w = eqb.eqb_gate_topk(z.cuda(), None, 8, renorm=False)
    want = ref.choose(z, None, 8)
    assert torch.equal(idx.cpu(), want)
    exact = ref.shares(z, want, "sigmoid", False, 1.0)
    assert torch.all((w.cpu().double() - exact).abs() <= 400 * U * exact + 4 * 2.0 ** -149)


@pytest.mark.parametrize("score,renorm", [("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_gradients_of_far_sigmoids(score, renorm, sign):
    """s (1 - s) is exp(-|z|) on either side; the gradients that come in bring it back into the normal range."""
    T, K, big = 64, 2, 2.0 ** 60
    z = sign * torch.linspace(80.0, 100.0, T * 8).view(T, 8)
    idx = torch.tensor([[1, 6]], dtype=torch.int32).repeat(T, 1)
    gw = torch.tensor([[1.0, -2.0]]).repeat(T, 1) * big
    got = eqb.eqb_gate_grad(z.cuda(), idx.cuda(), gw.cuda(), score=score, renorm=renorm).cpu().double()
    exact, size = ref.gate_grad(z, idx, gw, score, renorm, 1.0)
    # a factor below 2^-126 is off by up to two steps of 2^-149
    assert torch.all((got - exact).abs() <= 500 * U * size + 8 * big * 2.0 ** -149)
