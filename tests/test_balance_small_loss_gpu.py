"""The balance loss where the lists name experts of little probability: a sum of
non-negative terms, so 1e-5 of itself however small it is."""
import numpy as np
import pytest
import torch

from test_balance_loss_gpu import run
from train_reference import balance

pytestmark = pytest.mark.gpu


# one to a few tokens a microbatch, a cluster a microbatch; 6,000 and more: blocks over all of them
@pytest.mark.parametrize("T,M", [(1, 1), (6, 6), (90, 2), (6000, 900), (30000, 3)])
@pytest.mark.parametrize("E", [8, 128, 512])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("grad", ["none", "fp32"])
def test_lists_of_unlikely_experts(T, M, E, score, grad):
    rng = np.random.default_rng(T + E)
    z = rng.standard_normal((T, E)).astype(np.float32)
    z[:, 0] += 12.0
    z[:, 1:4] -= 12.0
    z = torch.from_numpy(z)
    idx = np.tile(np.array([[1, 3]], np.int32), (T, 1))
    off = np.array([T * l // M for l in range(M + 1)], np.int64)
    counts, loss, prob, g, _, err = run(z, idx, off, None, score, 0.5, 0.0, grad, rng=rng)
    if T <= 6000:
        want, r_counts = balance(z.double().numpy(), idx, off, score, 0.5, 0.0)[:2]
        want = want[:, 0]
        assert np.array_equal(counts, r_counts)
    else:
        zz = z.double()
        p = torch.softmax(zz, 1) if score == "softmax" else torch.sigmoid(zz) / torch.sigmoid(zz).sum(1, keepdim=True)
        want = np.array([0.5 * (p[a:b, 1].mean() + p[a:b, 3].mean()).item() / 2 for a, b in zip(off, off[1:])])
    assert err == 0
    assert np.all(np.abs(loss[:, 0] - want) <= 1e-5 * want), (loss[:3, 0], want[:3])
