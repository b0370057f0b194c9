"""eqb_balance_loss with logits far from zero, the types' lowest and largest values among them.

Against the 64-bit plain form.  A probability is off by less than 1e-5 of itself:
a difference of two logits is rounded once (2^-24 of it), and those that matter
are within 100 of the row's largest, where that is 100 * 2^-24 log2(e) < 9e-6.  A
gradient is p_j (R_j - sum p_e R_e) with R = F - 1/E: the sum is off by 1e-5 of
sum p_e |R_e|, whose terms may cancel, and each factor by 1e-5 of itself, so 2e-5
of the terms in all, beside the roundings of grad_in and of the output."""
import numpy as np
import pytest
import torch

from test_balance_loss_gpu import make, run
from train_reference import balance, probabilities

pytestmark = pytest.mark.gpu


def lowest(dtype):
    return torch.finfo(dtype).min


def terms(z, idx, off, counts, score, alpha, zeta):
    """The magnitude [T,E] of what a gradient is the sum of."""
    T, E = z.shape
    size = np.zeros((T, E))
    for l in range(len(off) - 1):
        n = off[l + 1] - off[l]
        R = np.abs(counts[l] / (idx.shape[1] * max(n, 1)) - 1 / E)
        for t in range(off[l], off[l + 1]):
            p, lse, s = probabilities(z[t], score)
            size[t] = alpha / n * p * (R + p @ R) + 2 * zeta / n * p * abs(lse)
            if score == "sigmoid":
                size[t] *= 1 - s
    return size


def check(z, idx, off, score, alpha, zeta, out, bf16=False):
    counts, loss, prob, grad, gi, err = out
    zz = z.double().numpy()
    r_loss, r_counts, r_prob, r_grad, _ = balance(zz, idx, off, score, alpha, zeta)
    assert err == 0
    assert np.array_equal(counts, r_counts)
    assert np.all(np.abs(loss - r_loss) <= 1e-5 * np.abs(r_loss))
    assert np.all(np.abs(prob - r_prob) <= 1e-5 * r_prob + 1e-30)
    if grad is None:
        return
    want = r_grad + (0.0 if gi is None else gi.astype(np.float64))
    tol = 2e-5 * terms(zz, idx, off, r_counts, score, alpha, zeta) + 2.0 ** -22 * np.abs(want) + 1e-30
    if gi is not None:
        tol += 2.0 ** -23 * np.abs(gi)
    if bf16:
        tol = tol * 1.01 + 2.0 ** -8 * np.abs(want)
    bad = np.abs(grad - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:3], grad[bad][:3], want[bad][:3])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [8, 96, 128, 256, 1024])
@pytest.mark.parametrize("grad,add", [("none", False), ("fp32", True), ("bf16", False)])
def test_closed_by_the_lowest_value(dtype, score, E, grad, add):
    """Experts, and all experts of a token, closed by the type's lowest value:
    such a row's probabilities are equal."""
    z, idx, off, mask, rng = make(90, E, 2, 3, E, dtype=dtype)
    z[::4, 1:5] = lowest(dtype)
    z[7] = lowest(dtype)
    z[40:44] = lowest(dtype)
    z[50] = -float("inf")
    z[50, 2:4] = lowest(dtype)  # what is left beside closed ones
    out = run(z, idx, off, mask, score, 0.1, 0.0, grad, add, rng=rng)
    check(z, idx, off, score, 0.1, 0.0, out, bf16=grad == "bf16")


@pytest.mark.parametrize("score,shift", [("softmax", s) for s in (-3e38, -1e12, -2e9, -1e7, -2.0 ** 20, 1e7, 2e9, 1e12, 3e38)] +
                         [("sigmoid", s) for s in (-3e38, -1e12, -2e9, -1e7, -2.0 ** 20)])
def test_rows_far_from_zero(score, shift):
    """fp32 rows around a common value, beside rows near zero in the same warps."""
    z, idx, off, mask, rng = make(64, 64, 4, 2, 11, dtype=torch.float32)
    z[1::4] += shift
    z[2::4] = shift
    z[3::4, :8] = shift
    zeta = 1e-3 if score == "softmax" and abs(shift) < 1e15 else 0.0
    check(z, idx, off, score, 0.1, zeta, run(z, idx, off, mask, score, 0.1, zeta, rng=rng))
