"""Parameters whose gradient has been zero so far stay what they are, at the
smallest eps that is taken too."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [600, 513])  # whole units and a tail
def test_idle_parameters(bits, n):
    p = torch.full((n,), 0.5, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    opt = eqb.EqbAdamW([p], state_bits=bits)
    opt.step([torch.zeros(n, device="cuda")], lr=1e-2, step=1, eps=2.0 ** -126, weight_decay=0.0, err_flag=err)
    assert torch.equal(p, torch.full_like(p, 0.5)) and err.item() == 0
    for eps in (1e-39, 1e-46):
        with pytest.raises(eqb.EqbError):
            opt.step([torch.zeros(n, device="cuda")], lr=1e-2, step=1, eps=eps, weight_decay=0.0)
    assert torch.equal(p, torch.full_like(p, 0.5))
