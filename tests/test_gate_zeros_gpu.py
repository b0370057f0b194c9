"""eqb_gate_topk where scores are zeros of both signs: -0 and +0 are equal, so the
lower expert comes first, whatever the number of tokens.  c = z + b is -0 only where
both are."""
import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


def zeros(T, E, seed, ones):
    g = torch.Generator().manual_seed(seed)
    z = torch.where(torch.rand(T, E, generator=g) < 0.5, 0.0, -0.0)
    if ones:  # a few above and below, so that the zeros are the list's end
        u = torch.rand(T, E, generator=g)
        z = torch.where(u < 2.0 / E, 1.0, torch.where(u > 0.9, -1.0, z))
    b = torch.zeros(E)
    b[torch.randperm(E, generator=g)[:E // 3]] = -0.0
    return z, b


@pytest.mark.parametrize("E,groups,top_groups,K", [(8, 1, 1, 3), (40, 1, 1, 6), (64, 1, 1, 8), (96, 4, 2, 8), (128, 8, 4, 8), (256, 1, 1, 8),
                                                   (256, 8, 4, 8), (512, 2, 1, 1), (520, 1, 1, 8), (256, 1, 1, 12)])
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("ones", [False, True])
def test_zeros_of_both_signs_are_ties(E, groups, top_groups, K, fp32, ones):
    T = 9000
    z, b = zeros(T, E, E + K, ones)
    z = z if fp32 else z.bfloat16()
    for bias in (b, torch.full((E,), -0.0)):
        want = ref.choose(z, bias, K, groups, top_groups, True)
        for part in (slice(0, T), slice(0, 4096)):  # a thread a token, where that serves the sizes, and a warp a token
            idx, _ = eqb.eqb_gate_topk(z[part].cuda(), bias.cuda(), K, groups=groups, top_groups=top_groups, group_score="top2")
            assert torch.equal(idx.cpu(), want[part])
