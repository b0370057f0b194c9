"""Plain 64-bit forms of a router's training operators (numpy, row by row from
the formulas): what the GPU tests compare the kernels with."""
from __future__ import annotations

import numpy as np


def counts_of(idx, offsets, E, mask):
    """f[l, e]: entries of the lists of microbatch l's valid tokens that name e."""
    M = len(offsets) - 1
    f = np.zeros((M, E), np.int64)
    for l in range(M):
        for t in range(offsets[l], offsets[l + 1]):
            if mask[t]:
                for e in idx[t]:
                    if 0 <= e < E:
                        f[l, e] += 1
    return f


def probabilities(z, score):
    """p [E], lse and sigmoids of one row; zeros for a row without a finite logit."""
    z = np.asarray(z, np.float64)
    if not np.any(z > -np.inf):
        return np.zeros_like(z), 0.0, np.zeros_like(z)
    top = z.max()
    e = np.exp(z - top)
    lse = top + np.log(e.sum())
    if score == "softmax":
        return e / e.sum(), lse, None
    with np.errstate(over="ignore"):
        s = 1.0 / (1.0 + np.exp(-z))
        # relative to a reference, so that a row of very negative logits keeps its ratios
        ref = min(top, 0.0)
        r = 1.0 / (np.exp(ref) + np.exp(ref - z))
    return r / r.sum(), lse, s


def balance(z, idx, offsets, score, alpha, zeta, mask=None, counts=None):
    """loss [M,2], counts [M,E], prob [M,E], gradient [T,E] (F constant), and
    the magnitude [T,E] of the terms that the gradient is the sum of."""
    T, E = z.shape
    K = idx.shape[1]
    M = len(offsets) - 1
    mask = np.ones(T, bool) if mask is None else np.asarray(mask, bool)
    f = counts_of(idx, offsets, E, mask) if counts is None else counts
    loss, prob = np.zeros((M, 2)), np.zeros((M, E))
    grad, size = np.zeros((T, E)), np.zeros((T, E))
    for l in range(M):
        rows = [t for t in range(offsets[l], offsets[l + 1]) if mask[t]]
        n = len(rows)
        if not n:
            continue
        F = f[l] / (K * n)
        for t in rows:
            p, lse, s = probabilities(z[t], score)
            prob[l] += p / n
            loss[l, 1] += zeta * lse * lse / n
            g = alpha / n * p * (F - p @ F)
            size[t] = alpha / n * p * (np.abs(F - 1 / E) + np.abs(p @ F - p.sum() / E) + 1e-6 / E) + 2 * zeta / n * p * abs(lse)
            if score == "sigmoid":
                g, size[t] = g * (1 - s), size[t] * (1 - s)
            grad[t] = g + 2 * zeta / n * lse * p
        loss[l, 0] = alpha * (F @ prob[l])
    return loss, f, prob, grad, size


def adamw(p, g, m, v, lr, step, beta1, beta2, eps, wd):
    """New p, m, v in 64 bits."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    upd = lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p - lr * wd * p - upd, m, v
