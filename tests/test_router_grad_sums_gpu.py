"""dW's sums over many tokens of one sign, where what the tensor cores cut off adds up.

512 tokens are 32 MMAs into one fp32 sum S.  An MMA cuts off at most a last place,
2^-23 of the sum so far: 2^-23 S (1 + 2 + ... + 32) / 32 = 16.5 * 2^-23 S = 2.0e-6 S
at most, half of it in the mean.  The sums of 512 are added up rounded to nearest
(2^-24 of the sum so far each): 43 of them at most in a block here, 22 * 2^-24 in
the worst case, and up to 12 blocks' sums, 12 * 2^-24: 2.0e-6 in all, without
a bias.  So 4e-6 for every element and 1.2e-6 for the mean of the signed errors;
one sum over the 7,000 to 22,000 tokens of a block is off by 7e-6 to 2e-5."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,E,dx,add", [(65536, 4096, 128, False, False), (65536, 4096, 128, True, True), (65536, 2048, 256, False, False),
                                          (131072, 1024, 64, True, False)])
def test_sums_of_one_sign(T, d, E, dx, add):
    g = torch.Generator(device="cuda").manual_seed(T + d)
    dz = (0.5 + torch.rand(T, E, generator=g, device="cuda")).bfloat16()
    x = (0.5 + torch.rand(T, d, generator=g, device="cuda")).bfloat16()
    W = torch.zeros(E, d, dtype=torch.bfloat16, device="cuda")
    dW = torch.rand(E, d, generator=g, device="cuda")
    want = dz.double().t() @ x.double()
    if add:
        want += dW.double()
    out = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda") if dx else None
    eqb.eqb_router_grad(dz, x, W, dx=out, dW=dW, accumulate_dx=add, accumulate_dW=add)
    off = (dW.double() - want) / want
    print("largest %.2e, mean %.2e" % (off.abs().max().item(), off.mean().item()))
    assert off.abs().max().item() <= 4e-6
    assert abs(off.mean().item()) <= 1.2e-6
