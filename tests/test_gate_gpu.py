"""eqb_gate_topk and eqb_gate_grad against 64 bits.

The choice is exact.  A weight is a quotient of exponentials: each within 4 ulps of
its argument's, whose rounding moves it by |z - m| 2^-24 (twice, where a base change is
rounded too), and a sum of up to 1,024 of them, 32 a lane, in at most 32 + 5 + 2 additions
and as many rescalings: (2 * 39 + 24 + 2 range) 2^-24 of the weight, and one subnormal
step.  A gradient is a sum of at most K + 2 such terms."""
import math

import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def logits(T, E, fp32, seed, wide=1.0, closed=True):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(T, E, generator=g) * wide
    if closed and T > 3:
        z[1, E // 2:] = -math.inf   # half the experts
        z[2] = -math.inf            # all of them
        z[3, 1:] = -math.inf        # all but one
    z = z if fp32 else z.bfloat16()
    return z, torch.randn(E, generator=g) * 0.2


def run(z, b, K, idx_only=False, **kw):
    T = z.shape[0]
    idx = Guarded((T, K), torch.int32, fill=-7)
    w = Guarded((T, K), torch.float32, fill=-7.0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    mask = kw.pop("mask", None)
    eqb.eqb_gate_topk(z.cuda(), None if b is None else b.cuda(), K, mask=None if mask is None else mask.cuda(), topk_idx=idx.view,
                      weight=w.view, err_flag=err, **kw)
    torch.cuda.synchronize()
    assert idx.intact() and w.intact()
    return idx.view.cpu(), w.view.cpu(), err.item()


def check(z, b, K, score, renorm, scale, groups=1, top_groups=1, top2=False, mask=None):
    idx, w, err = run(z, b, K, score=score, renorm=renorm, scale=scale, groups=groups, top_groups=top_groups,
                      group_score="top2" if top2 else "max", mask=mask)
    assert err == 0
    want = ref.choose(z, b, K, groups, top_groups, top2, mask)
    assert torch.equal(idx, want)
    exact = ref.shares(torch.where(torch.isfinite(z), z, torch.tensor(-math.inf).to(z.dtype)), want, score, renorm, scale)
    fin = z.double()[torch.isfinite(z)]
    spread = float(fin.max() - fin.min()) + float(fin.abs().max()) if fin.numel() else 0.0
    assert torch.all((w.double() - exact).abs() <= (102 + 2 * spread) * U * exact.abs() + abs(scale) * 2.0 ** -148), \
        ((w.double() - exact).abs() / exact.abs()).nan_to_num(0).max()


@pytest.mark.parametrize("E,K", [(8, 1), (8, 2), (16, 7), (40, 6), (64, 8), (72, 8), (96, 1), (128, 8), (256, 8), (256, 31), (264, 6),
                                 (512, 8), (520, 12), (1000, 8), (1024, 31)])
@pytest.mark.parametrize("score,renorm", [("sigmoid", True), ("softmax", False)])
@pytest.mark.parametrize("fp32", [False, True])
def test_without_groups(E, K, score, renorm, fp32):
    z, b = logits(67, E, fp32, E + K)
    check(z, b, K, score, renorm, 2.5)


@pytest.mark.parametrize("E,groups,top_groups,K", [(8, 4, 2, 2), (16, 8, 3, 6), (16, 16, 5, 4), (40, 8, 4, 6), (64, 8, 4, 8), (96, 32, 4, 8),
                                                   (128, 8, 1, 8), (256, 8, 4, 8), (256, 32, 7, 6), (256, 3 + 1, 3, 31), (384, 3, 2, 8),
                                                   (1024, 8, 4, 8), (1000, 5, 2, 12)])
@pytest.mark.parametrize("top2", [False, True])
@pytest.mark.parametrize("score,renorm", [("sigmoid", False), ("softmax", True)])
def test_groups(E, groups, top_groups, K, top2, score, renorm):
    z, b = logits(70, E, False, E * groups)
    check(z, b, K, score, renorm, 1.0, groups, top_groups, top2)


@pytest.mark.parametrize("T,E,K,groups", [(1, 256, 8, 8), (2, 128, 8, 1), (31, 64, 6, 8), (4097, 256, 8, 8), (20011, 128, 8, 1),
                                          (20011, 256, 8, 8), (70001, 64, 2, 4), (9001, 512, 8, 8), (9001, 40, 6, 8), (9001, 1000, 8, 1),
                                          (40003, 96, 8, 8)])
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("score,renorm", [("sigmoid", True), ("softmax", False)])
def test_many_tokens(T, E, K, groups, fp32, score, renorm):
    z, b = logits(T, E, fp32, T)
    g = torch.Generator().manual_seed(T)
    mask = torch.rand(T, generator=g) < 0.8
    z[~mask] = math.nan
    mask[2:4] = True
    z[2:3] = -math.inf
    z[3:4] = 0.0
    check(z, b, K, score, renorm, 1.0, groups, max(1, groups // 2), True, mask)


def test_ties_go_to_the_lower_expert_and_group():
    """Few different values, zeros of both signs, and no bias."""
    g = torch.Generator().manual_seed(1)
    for E, groups, top_groups, K in ((64, 1, 1, 8), (256, 8, 4, 8), (40, 8, 3, 6), (512, 16, 4, 12)):
        z = torch.randint(-1, 2, (9000, E), generator=g).float()
        z = torch.where(torch.rand(z.shape, generator=g) < 0.5, z, -z)  # -0 among them
        z[:50] = 0.0
        z[50:99] = -0.0
        check(z.bfloat16(), None, K, "sigmoid", True, 1.0, groups, top_groups, True)
        check(z, None, K, "sigmoid", True, 1.0, groups, top_groups, False)


def test_closed_by_the_bias():
    z, b = logits(300, 64, False, 3, closed=False)
    b[5:60] = -math.inf
    idx, w, err = run(z, b, 12, score="sigmoid")
    assert err == 0 and torch.equal(idx, ref.choose(z, b, 12))
    assert (idx[:, 9:] == -1).all() and not w[:, 9:].any() and torch.all((w.sum(1) - 1).abs() < 1e-6)


def test_closed_second_of_a_group_counts_nothing():
    z = torch.full((64, 16), -math.inf)
    z[:, 0], z[:, 1] = 1.0, 0.5      # group 0: 1.5
    z[:, 4] = 2.0                    # group 1: 2 alone
    z[:, 8], z[:, 9] = -3.0, -3.0    # group 2: -6
    idx, w, _ = run(z, None, 2, groups=4, top_groups=1, group_score="top2", renorm=False, score="softmax")
    assert torch.equal(idx, torch.tensor([[4, -1]], dtype=torch.int32).repeat(64, 1)) and not w[:, 1].any()


@pytest.mark.parametrize("level", [-300.0, -89.0, 60.0, 300.0])
def test_far_logits_keep_their_shares(level):
    """Sigmoids that underflow in fp32 are renormalised all the same."""
    g = torch.Generator().manual_seed(9)
    z = (torch.randn(200, 64, generator=g) + level)
    check(z, None, 8, "sigmoid", True, 2.5)
    check(z, None, 8, "softmax", True, 1.0)
    check(z, None, 8, "softmax", False, 1.0)
    check(z, None, 8, "sigmoid", False, 1.0)


@pytest.mark.parametrize("T", [40, 9000])
@pytest.mark.parametrize("fp32", [False, True])
def test_nonfinite_raises_the_flag(T, fp32):
    for bad in (math.nan, math.inf):
        z, b = logits(T, 128, fp32, 4)
        z[T - 7, 77] = bad
        idx, _, err = run(z, b, 8)
        assert err == 4 and idx.min() >= -1 and idx.max() < 128
        keep = torch.arange(T) != T - 7
        assert torch.equal(idx[keep], ref.choose(z[keep], b, 8))
        mask = keep.clone()
        assert run(z, b, 8, mask=mask)[2] == 0  # nobody looks at it
    z, b = logits(T, 128, fp32, 4)
    b[3] = math.nan
    assert run(z, b, 8)[2] == 4


def test_no_tokens_and_made_outputs():
    idx, w = eqb.eqb_gate_topk(torch.empty(0, 64, device="cuda"), None, 8)
    assert idx.shape == (0, 8) and w.shape == (0, 8)
    z, b = logits(100, 64, True, 5)
    idx, w = eqb.eqb_gate_topk(z.cuda(), b.cuda(), 8, mask=torch.ones(100, dtype=torch.uint8, device="cuda"))
    assert torch.equal(idx.cpu(), ref.choose(z, b, 8))
    again = eqb.eqb_gate_topk(z.cuda(), b.cuda(), 8)
    assert torch.equal(again[0], idx) and torch.equal(again[1], w)


def test_agrees_with_the_routing():
    """Without groups the choice is eqb_route_topk's."""
    z, b = logits(5000, 256, False, 6, closed=False)
    idx, _, _ = run(z, b, 8)
    want = torch.empty(5000, 8, dtype=torch.int32, device="cuda")
    eqb.eqb_route_topk(z.cuda(), b.cuda(), 8, topk_idx=want)
    assert torch.equal(idx, want.cpu())


# ---- the gradient

def lists(T, E, K, seed, drop=0.2):
    g = torch.Generator().manual_seed(seed)
    idx = torch.argsort(torch.rand(T, E, generator=g), dim=1)[:, :K].int()
    idx[torch.rand(T, K, generator=g) < drop] = -1
    idx[0] = -1
    if T > 5:
        idx[4, 0], idx[5, -1] = E, -2 ** 31  # names no expert
    return idx, torch.randn(T, K, generator=g)


def run_grad(z, idx, gw, score, renorm, scale, grad_in=None, bf16=False, in_place=False):
    T, E = z.shape
    out = Guarded((T, E), torch.bfloat16 if bf16 else torch.float32, fill=5.0, canary=-3.0)
    gi = None
    if grad_in is not None:
        if in_place:
            out.view.copy_(grad_in)
            gi = out.view
        else:
            gi = grad_in.cuda()
    eqb.eqb_gate_grad(z.cuda(), idx.cuda(), gw.cuda(), score=score, renorm=renorm, scale=scale, grad_in=gi, grad_out=out.view)
    torch.cuda.synchronize()
    assert out.intact()
    return out.view.cpu()


KINDS = [("sigmoid", True), ("sigmoid", False), ("softmax", True), ("softmax", False)]


def within(got, z, idx, gw, score, renorm, scale, grad_in, bf16):
    want, size = ref.gate_grad(z, idx, gw, score, renorm, scale)
    K = idx.shape[1]
    fin = z.double()[torch.isfinite(z)]
    spread = float(fin.max() - fin.min()) + float(fin.abs().max())
    tol = (102 + 2 * spread + 4 * K) * U * size + 2.0 ** -140
    if grad_in is not None:
        want = want + grad_in.double()
        tol = tol + U * want.abs()
    if bf16:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    assert torch.all((got.double() - want).abs() <= tol)


@pytest.mark.parametrize("score,renorm", KINDS)
@pytest.mark.parametrize("E,K,fp32", [(8, 2, False), (16, 1, True), (40, 6, False), (64, 8, True), (128, 8, False), (256, 8, True),
                                      (264, 31, False), (512, 8, False), (1000, 6, True), (1024, 31, False)])
@pytest.mark.parametrize("T", [1, 65])
def test_gradient(score, renorm, E, K, fp32, T):
    z, _ = logits(T, E, fp32, E, closed=False)
    idx, gw = lists(T, E, K, E)
    g = torch.Generator().manual_seed(2)
    gi = torch.randn(T, E, generator=g)
    within(run_grad(z, idx, gw, score, renorm, 2.5), z, idx, gw, score, renorm, 2.5, None, False)
    within(run_grad(z, idx, gw, score, renorm, 1.0, gi), z, idx, gw, score, renorm, 1.0, gi, False)
    within(run_grad(z, idx, gw, score, renorm, 1.0, gi, in_place=True), z, idx, gw, score, renorm, 1.0, gi, False)
    within(run_grad(z, idx, gw, score, renorm, 1.0, gi, bf16=True), z, idx, gw, score, renorm, 1.0, gi, True)
    within(run_grad(z, idx, gw, score, renorm, -1.0, None, bf16=True), z, idx, gw, score, renorm, -1.0, None, True)


@pytest.mark.parametrize("score,renorm", KINDS)
@pytest.mark.parametrize("E", [64, 128, 256])
def test_gradient_of_many_tokens(score, renorm, E):
    T = 30011
    z, _ = logits(T, E, False, E, closed=False)
    idx, gw = lists(T, E, 8, E)
    within(run_grad(z, idx, gw, score, renorm, 1.0), z, idx, gw, score, renorm, 1.0, None, False)


@pytest.mark.parametrize("score,renorm", KINDS)
def test_gradient_of_an_expert_named_twice(score, renorm):
    z, _ = logits(50, 32, True, 8, closed=False)
    idx, gw = lists(50, 32, 6, 3, drop=0.1)
    idx[:, 3] = idx[:, 0]
    idx[::2, 5] = idx[::2, 0]
    within(run_grad(z, idx, gw, score, renorm, 1.0), z, idx, gw, score, renorm, 1.0, None, False)


@pytest.mark.parametrize("score,renorm", KINDS)
def test_rows_without_a_list_are_not_looked_at(score, renorm):
    z, _ = logits(40, 64, False, 8, closed=False)
    idx, gw = lists(40, 64, 4, 3)
    idx[10:20] = -1
    z[10:20] = math.nan
    gw[10:20] = math.nan
    got = run_grad(z, idx, gw, score, renorm, 1.0)
    assert not got[10:20].any() and torch.isfinite(got).all()
    gi = torch.randn(40, 64)
    got = run_grad(z, idx, gw, score, renorm, 1.0, gi, in_place=True)
    assert torch.equal(got[10:20], gi[10:20])


@pytest.mark.parametrize("score,renorm", KINDS)
def test_closed_experts_have_no_gradient(score, renorm):
    z, _ = logits(40, 64, False, 8, closed=False)
    idx, gw = lists(40, 64, 4, 3)
    shut = torch.ones(40, 64, dtype=torch.bool).scatter_(1, idx.clamp(0, 63).long(), False)
    z[shut & (torch.rand(40, 64) < 0.5)] = -math.inf
    got = run_grad(z, idx, gw, score, renorm, 1.0)
    assert not got[torch.isinf(z)].any()
    within(got, z, idx, gw, score, renorm, 1.0, None, False)


@pytest.mark.parametrize("score,renorm", KINDS)
def test_gradient_against_differences(score, renorm):
    """(L(z + h v) - L(z - h v)) / 2h of L = sum g w, in 64 bits: off by h^2 |v|^3 L''' / 6 < 2e-7 of the terms for h = 1e-4."""
    T, E, K = 20, 32, 5
    z, _ = logits(T, E, True, 11, closed=False)
    idx, gw = lists(T, E, K, 12)
    got = run_grad(z, idx, gw, score, renorm, 1.5)
    v = torch.randn(T, E, dtype=torch.float64)
    loss = lambda x: (ref.shares(x, idx, score, renorm, 1.5) * gw.double()).sum(1)  # noqa: E731
    h = 1e-4
    diff = (loss(z.double() + h * v) - loss(z.double() - h * v)) / (2 * h)
    size = (ref.gate_grad(z, idx, gw, score, renorm, 1.5)[1] * v.abs()).sum(1)
    assert torch.all(((got.double() * v).sum(1) - diff).abs() <= 2e-5 * size + 1e-9)


def test_gradient_in_a_graph_with_the_gate():
    """Captured and replayed on other inputs, on a stream of its own."""
    z, b = (t.cuda() for t in logits(3000, 128, False, 7, closed=False))
    gw = torch.randn(3000, 8, device="cuda")
    idx, w = eqb.eqb_gate_topk(z, b, 8)
    dz = eqb.eqb_gate_grad(z, idx, gw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eqb.eqb_gate_topk(z, b, 8, topk_idx=idx, weight=w)
        eqb.eqb_gate_grad(z, idx, gw, grad_out=dz)
    z.copy_(logits(3000, 128, False, 8, closed=False)[0])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(idx.cpu(), ref.choose(z.cpu(), b.cpu(), 8))
    within(dz.cpu(), z.cpu(), idx.cpu(), gw.cpu(), "sigmoid", True, 1.0, None, False)
