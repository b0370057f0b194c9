"""The training calls launch on the current device: tensors of another one are refused."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


def test_tensors_of_another_device_are_refused(monkeypatch):
    z = torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda:0")
    x = torch.zeros(8, 128, dtype=torch.bfloat16, device="cuda:0")
    W = torch.zeros(64, 128, dtype=torch.bfloat16, device="cuda:0")
    idx = torch.zeros(8, 2, dtype=torch.int32, device="cuda:0")
    off = torch.tensor([0, 8], device="cuda:0")
    dx, dW = torch.full_like(x, 3.0), torch.full((64, 128), 3.0, device="cuda:0")
    counts = torch.full((1, 64), 7, dtype=torch.int32, device="cuda:0")
    p = torch.ones(64, device="cuda:0")
    opt = eqb.EqbAdamW([p])
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        with pytest.raises(ValueError, match="current device"):
            eqb.eqb_balance_loss(z, idx, off, 0.1, counts=counts)
        with pytest.raises(ValueError, match="current device"):
            eqb.eqb_router_grad(z, x, W, dx=dx, dW=dW)
        with pytest.raises(ValueError, match="current device"):
            opt.step([torch.ones(64, device="cuda:0")], lr=1e-3, step=1)
    torch.cuda.synchronize()
    assert bool((dx == 3.0).all()) and bool((dW == 3.0).all()) and bool((counts == 7).all()) and bool((p == 1.0).all())
    eqb.EqbAdamW([]).step([], lr=1e-3, step=1)  # nothing to do
