"""EqbAdamW beside autograd: what a step writes counts as modified in place."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_raises_the_versions_of_what_it_writes(bits):
    p = [torch.nn.Parameter(torch.ones(n, device="cuda")) for n in (300, 20, 5)]
    c = [torch.zeros(300, dtype=torch.bfloat16, device="cuda"), None, torch.zeros(5, dtype=torch.bfloat16, device="cuda")]
    opt = eqb.EqbAdamW(p, state_bits=bits, copies=c)
    seen = [t._version for t in p], c[0]._version, c[2]._version
    opt.step([torch.ones(300, device="cuda"), torch.ones(20, device="cuda"), None], lr=1e-3, step=1)
    assert p[0]._version > seen[0][0] and p[1]._version > seen[0][1] and c[0]._version > seen[1]
    assert p[2]._version == seen[0][2] and c[2]._version == seen[2]  # no gradient: left as they are


def test_backward_through_a_value_that_is_gone_is_refused():
    w = torch.nn.Parameter(torch.randn(64, 32, device="cuda"))
    opt = eqb.EqbAdamW([w])
    loss = (w * w).sum()  # saves w
    (g,) = torch.autograd.grad(loss, [w], retain_graph=True)
    opt.step([g], lr=1e-3, step=1)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    (w * w).sum().backward()  # a new graph is fine
    assert torch.equal(w.grad, 2 * w.detach())


def test_parameters_made_in_inference_mode():
    with torch.inference_mode():
        p = torch.ones(8, device="cuda")
        eqb.EqbAdamW([p]).step([torch.ones(8, device="cuda")], lr=1e-2, step=1, weight_decay=0.0)
    assert torch.allclose(p, torch.full_like(p, 0.99))


def test_views_of_one_buffer():
    flat = torch.ones(600, device="cuda")
    p = list(flat.split([100, 200, 300]))
    opt = eqb.EqbAdamW(p)
    x = torch.ones(200, device="cuda", requires_grad=True)
    loss = (p[1] * x).sum()  # saves the view
    opt.step([torch.ones(100, device="cuda"), torch.ones(200, device="cuda"), torch.ones(300, device="cuda")], lr=1e-3, step=1)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
