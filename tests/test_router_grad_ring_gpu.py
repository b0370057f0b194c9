"""dx added to, where a block fills every stage of its ring of old values many
times over: a stage that was refilled too early would show as a sum of another
tile.  Whole numbers, so every element is compared exactly."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


# rings of 3, 5, 6 and 6 stages, each of them used nine times or more
@pytest.mark.parametrize("T,d,E", [(33000, 1024, 256), (66001, 1024, 128), (50000, 1536, 48), (150000, 512, 16)])
@pytest.mark.parametrize("both", [False, True])
def test_added_to_through_a_ring_used_many_times(T, d, E, both):
    """dx alone, and beside dW in the shared launch; three calls on other old values."""
    g = torch.Generator(device="cuda").manual_seed(T)

    def whole(n, m, top):
        return torch.randint(-top, top + 1, (n, m), generator=g, device="cuda", dtype=torch.int16).bfloat16()

    dz, x, W = whole(T, E, 1), whole(T, d, 1), whole(E, d, 2)
    product = dz.float() @ W.float()
    dW = torch.empty(E, d, device="cuda") if both else None
    ws = torch.empty(eqb.eqb_router_grad_workspace_bytes(T, d, E), dtype=torch.uint8, device="cuda") if both else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(3):
        dx = whole(T, d, 100)
        want = (product + dx.float()).bfloat16()  # below 2^24: one rounding either way
        eqb.eqb_router_grad(dz, x, W, dx=dx, dW=dW, accumulate_dx=True, workspace=ws, err_flag=err)
        assert torch.equal(dx, want)
    assert err.item() == 0
