"""eqb_expert_wgrad added to what is there: an expert without blocks is left as it is,
bit for bit (-0 and NaN payloads among it)."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


@pytest.mark.parametrize("blk,n,d", [([2, 0, 3], 144, 272), ([0, 1], 16, 16), ([0, 0, 0], 272, 528), ([1, 0] * 40, 128, 256), ([0, 2, 0], 400, 1040)])
def test_experts_without_blocks_are_left_as_they_are(blk, n, d):
    g = torch.Generator(device="cuda").manual_seed(n)
    P, E = max(sum(blk), 1), len(blk)
    a = torch.randint(-2, 3, (n, P * 128), generator=g, device="cuda").float().to(E4M3)
    b = torch.randint(-3, 4, (d, P * 128), generator=g, device="cuda").float().to(E4M3)
    sa, sb = torch.ones(P, n, device="cuda"), torch.ones(P, d, device="cuda")
    blocks = torch.tensor([0] + blk).cumsum(0).int().cuda()
    before = torch.tensor([-2 ** 31, 0x7fc12345, 0x3f800000, 1], dtype=torch.int32, device="cuda").repeat(n * d // 4).view(n, d)
    dW = Guarded((E, n, d), torch.float32)
    for e in range(E):
        if blk[e]:
            dW.view[e] = e + 1.0
        else:
            dW.view[e].view(torch.int32).copy_(before)
    eqb.eqb_expert_wgrad(a, sa, b, sb, blocks, dW=dW.view, accumulate=True)
    torch.cuda.synchronize()
    assert dW.intact()
    for e in range(E):
        if blk[e]:
            at = slice(128 * int(blocks[e]), 128 * int(blocks[e + 1]))
            assert torch.equal(dW.view[e], a[:, at].float() @ b[:, at].float().t() + (e + 1.0))
        else:
            assert torch.equal(dW.view[e].view(torch.int32), before)
    got = eqb.eqb_expert_wgrad(a, sa, b, sb, blocks, dW=dW.view)  # written: zeros
    assert all(not got[e].view(torch.int32).any() for e in range(E) if not blk[e])
