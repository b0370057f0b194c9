"""eqb_gate_grad added to in place gives the bits that it gives out of place: what a
token's lanes read of the row is read before any of them writes it."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("score,renorm", [("sigmoid", True), ("sigmoid", False), ("softmax", True), ("softmax", False)])
@pytest.mark.parametrize("E,K", [(8, 7), (64, 8), (128, 8), (256, 8), (264, 31), (512, 10), (1024, 31)])
@pytest.mark.parametrize("fp32", [False, True])
def test_in_place_and_out_of_place(score, renorm, E, K, fp32):
    T = 30011
    g = torch.Generator(device="cuda").manual_seed(E + K)
    z = torch.randn(T, E, generator=g, device="cuda")
    z = z if fp32 else z.bfloat16()
    idx = torch.randint(-1, E, (T, K), generator=g, device="cuda", dtype=torch.int32)  # some twice, some none
    gw, gi = torch.randn(T, K, generator=g, device="cuda"), torch.randn(T, E, generator=g, device="cuda")
    want = eqb.eqb_gate_grad(z, idx, gw, score=score, renorm=renorm, grad_in=gi)
    for _ in range(5):
        got = gi.clone()
        eqb.eqb_gate_grad(z, idx, gw, score=score, renorm=renorm, grad_in=got, grad_out=got)
        assert torch.equal(got, want)
