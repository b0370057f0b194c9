"""Plain 64-bit forms of the operators of the experts behind a router (torch on the
CPU, from the formulas): what the GPU tests compare the kernels with."""
from __future__ import annotations

import math

import torch

NINF = -math.inf


def choose(z, b, K, groups=1, top_groups=1, top2=False, mask=None):
    """int32 [T,K]: the chosen experts.  The sums that decide are fp32, as documented."""
    T, E = z.shape
    c = z.float() if b is None else z.float() + b
    if mask is not None:
        c = torch.where(mask[:, None], c, torch.tensor(NINF))
    if top_groups < groups:
        by = c.view(T, groups, -1)
        best = by.sort(2, descending=True).values
        score = best[:, :, 0].clone()
        if top2 and best.shape[2] > 1:
            score += torch.where(best[:, :, 1] > NINF, best[:, :, 1], torch.tensor(0.0))
        order = torch.argsort(-score, dim=1, stable=True)
        rank = torch.argsort(order, dim=1)
        c = torch.where((rank < top_groups)[:, :, None], by, torch.tensor(NINF)).reshape(T, E)
    idx = torch.argsort(-c, dim=1, stable=True)[:, :K]
    return torch.where(c.gather(1, idx) > NINF, idx, -1).int()


def shares(z, idx, score, renorm, scale):
    """Gate weights [T,K] in 64 bits; idx -1: 0."""
    z = z.double()
    here = (idx >= 0) & (idx < z.shape[1])
    zk = torch.where(here, z.gather(1, torch.where(here, idx, 0).long()), torch.tensor(NINF, dtype=torch.float64))
    if renorm:
        w = torch.softmax(torch.nn.functional.logsigmoid(zk) if score == "sigmoid" else zk, 1)
        w = torch.where(here.any(1, keepdim=True), w, torch.tensor(0.0, dtype=torch.float64))
    else:
        w = torch.sigmoid(zk) if score == "sigmoid" else torch.exp(zk - torch.logsumexp(z, 1, keepdim=True))
    return torch.where(here, w, torch.tensor(0.0, dtype=torch.float64)) * scale


def gate_grad(z, idx, g, score, renorm, scale):
    """The gradient [T,E] in 64 bits and the magnitude of the terms it is the sum of."""
    T, E = z.shape
    here = (idx >= 0) & (idx < E)
    at = torch.where(here, idx, 0).long()
    g = torch.where(here, g.double(), torch.tensor(0.0, dtype=torch.float64))
    w = shares(z, idx, score, renorm, 1.0)
    zk = z.double().gather(1, at)
    gb, size = (w * g).sum(1, keepdim=True), (w * g.abs()).sum(1, keepdim=True)
    out, mag = torch.zeros(T, E, dtype=torch.float64), torch.zeros(T, E, dtype=torch.float64)
    if score == "softmax" and not renorm:
        p = torch.softmax(z.double(), 1)
        out.scatter_add_(1, at, w * g)
        mag.scatter_add_(1, at, w * g.abs())
        out -= torch.where(here.any(1, keepdim=True), p * gb, torch.tensor(0.0, dtype=torch.float64))
        mag += torch.where(here.any(1, keepdim=True), p * size, torch.tensor(0.0, dtype=torch.float64))
    else:
        d, m = (w * (g - gb), w * (g.abs() + size)) if renorm else (w * g, w * g.abs())
        if score == "sigmoid":
            d, m = d * torch.sigmoid(-zk), m * torch.sigmoid(-zk)
        out.scatter_add_(1, at, torch.where(here, d, torch.tensor(0.0, dtype=torch.float64)))
        mag.scatter_add_(1, at, torch.where(here, m, torch.tensor(0.0, dtype=torch.float64)))
    return out * scale, mag * abs(scale)


def rows(idx, E):
    """offsets, blocks, slot and entry as lists."""
    T, K = idx.shape
    of = [[] for _ in range(E)]
    for i, e in enumerate(idx.flatten().tolist()):
        if 0 <= e < E:
            of[e].append(i)
    offsets, blocks, entry, slot = [0], [0], [], [-1] * (T * K)
    for r in of:
        for i in r:
            slot[i] = len(entry)
            entry.append(i)
        offsets.append(len(entry))
        blocks.append(blocks[-1] + (len(r) + 127) // 128)
    entry += [-1] * (T * K - len(entry))
    return offsets, blocks, slot, entry


def codes(x, dims):
    """Codes and scale of a block: x fp32, its largest magnitude over dims.  Operation by
    operation in fp32, as documented."""
    scale = x.abs().amax(dims, keepdim=True) * torch.tensor(1.0 / 448.0)
    scale = torch.where(scale < 2.0 ** -126, torch.tensor(0.0), scale)
    inv = torch.where(scale > 0, 1.0 / scale, torch.tensor(0.0))
    return (x * inv).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), scale


def spread(scale, dim, n):
    """A scale for each of n values from one for each 128 of them."""
    return scale.repeat_interleave(128, dim).narrow(dim, 0, n)
