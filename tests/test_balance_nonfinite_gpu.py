"""eqb_balance_loss: which logits raise the error flag.  One NaN in a token's
input makes all of its logits NaN."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu

NONFINITE = 4
NAN, INF = float("nan"), float("inf")


def flag(z, T, E, score, grad, mask=None):
    idx = torch.randint(0, E, (T, 2), dtype=torch.int32, device="cuda")
    off = torch.tensor([0, T // 3, T], device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.empty(T, E, device="cuda") if grad else None
    loss = eqb.eqb_balance_loss(z, idx, off, 0.1, score=score, mask=mask, grad_out=out, err_flag=err)[0]
    torch.cuda.synchronize()
    return err.item(), loss, out


# 70 tokens: a cluster a microbatch; 40,000: blocks over all of them
@pytest.mark.parametrize("T", [70, 40000])
@pytest.mark.parametrize("E", [8, 64, 200])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("grad", [False, True])
def test_rows_without_a_finite_logit(T, E, dtype, score, grad):
    z = torch.randn(T, E, device="cuda").to(dtype)
    row = T // 2
    z[row] = -INF  # closed: counts, has no probabilities and is no error
    code, loss, out = flag(z, T, E, score, grad)
    assert code == 0 and bool(loss.isfinite().all())
    assert out is None or (bool(out.isfinite().all()) and not out[row].any())
    for first in (0, 1, E - 1):  # NaN throughout, and beside -inf
        z[row] = NAN
        z[row, :first] = -INF
        assert flag(z, T, E, score, grad)[0] == NONFINITE
    z[row] = -INF
    z[row, E // 2] = NAN
    assert flag(z, T, E, score, grad)[0] == NONFINITE
    # a token that does not count raises nothing
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    mask[row] = False
    code, loss, out = flag(z, T, E, score, grad, mask)
    assert code == 0 and bool(loss.isfinite().all()) and (out is None or not out[row].any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_infinite_logits(dtype):
    z = torch.randn(50, 64, device="cuda").to(dtype)
    z[9, 3] = INF
    assert flag(z, 50, 64, "softmax", True)[0] == NONFINITE
    code, loss, out = flag(z, 50, 64, "sigmoid", True)  # its sigmoid is 1
    assert code == 0 and bool(loss.isfinite().all()) and bool(out.isfinite().all())
    z[9] = INF
    assert flag(z, 50, 64, "softmax", True)[0] == NONFINITE
