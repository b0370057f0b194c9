"""8-bit states over many steps beside 32-bit ones, in the range of beta2 that the
format is meant for (up to 0.95).

A code has three places of mantissa: its step is an eighth of it at most.  A
root whose change of a step is below half of that stays where it is, so roots
scatter around the true ones and at beta2 = 0.95 stand a little above them; both
within one step of a code.  m changes by a tenth of itself or more every step
and is only rounded, by half a step at most; some ten of those roundings are in
it at a time, of either sign: within an eighth too."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beta2", [0.9, 0.95])
@pytest.mark.parametrize("spread", [0.0, 1.0])  # of the sizes of a block's gradients, in logarithms
@pytest.mark.parametrize("late", [1.0, 0.1, 10.0])  # the gradients' size in the second half
def test_roots_stay_with_the_32_bit_ones(beta2, spread, late):
    g = torch.Generator(device="cuda").manual_seed(4)
    n, steps = 64 * 256, 2000
    size = torch.exp(spread * torch.randn(n, generator=g, device="cuda")) * 1e-3
    p8, p32 = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    o8, o32 = eqb.EqbAdamW([p8], state_bits=8), eqb.EqbAdamW([p32])
    for s in range(1, steps + 1):
        grad = torch.randn(n, generator=g, device="cuda") * size * (late if s > steps // 2 else 1.0)
        for o in (o8, o32):
            o.step([grad], lr=1e-4, step=s, beta2=beta2, weight_decay=0.0)
    root = o8.exp_avg_sq[0].float() * o8.sq_scale[0].repeat_interleave(256)
    ratio = (root / o32.exp_avg_sq[0].sqrt()).log()
    assert abs(ratio.mean().item()) <= 1 / 8
    assert ratio.std().item() <= 1 / 8
    m = o8.exp_avg[0].float() * o8.avg_scale[0].repeat_interleave(256)
    true = o32.exp_avg[0]
    assert ((m - true).square().mean() / true.square().mean()).sqrt().item() <= 1 / 8


def test_a_block_without_gradients_decays_by_its_scale():
    """Codes stay, the scale takes the decay: no root is left standing."""
    n, beta2 = 512, 0.95
    p = torch.zeros(n, device="cuda")
    opt = eqb.EqbAdamW([p], state_bits=8)
    opt.step([torch.rand(n, device="cuda") + 0.5], lr=0.0, step=1, beta2=beta2)
    codes, scale = opt.exp_avg_sq[0].clone(), opt.sq_scale[0].clone()
    for s in range(2, 102):
        opt.step([torch.zeros(n, device="cuda")], lr=0.0, step=s, beta2=beta2)
    assert torch.equal(codes.view(torch.uint8), opt.exp_avg_sq[0].view(torch.uint8))
    want = scale.double() * beta2 ** 50  # a hundred roots of beta2; four roundings a step
    assert torch.all((opt.sq_scale[0].double() - want).abs() <= 400 * 2.0 ** -24 * want)
