"""eqb_expert_combine and eqb_expert_combine_grad against 64 bits: a sum of K fused
multiply-adds (K 2^-24 of the magnitudes) rounded once to bf16 (2^-8); a dot product
of n exact products in at most n / 32 + 5 roundings on any path, so (n / 32 + 6) 2^-24 of the
magnitudes; a product rounded to fp32 and to bf16."""
import math

import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu


def case(T, n, K, E=8, drop=0.2, seed=0, more=0):
    g = torch.Generator().manual_seed(seed + T + n)
    idx = torch.randint(0, E, (T, K), generator=g, dtype=torch.int32)
    idx[torch.rand(T, K, generator=g) < drop] = -1
    if T > 1 and drop:
        idx[1] = -1
    _, _, slot, _ = ref.rows(idx, E)
    slot = torch.tensor(slot, dtype=torch.int32).view(T, K)
    rows = torch.randn(T * K + more, n, generator=g).bfloat16()
    rows[int((slot >= 0).sum()):] = math.nan  # rows of no slot are not read
    return rows, slot, torch.randn(T, K, generator=g), torch.randn(T, n, generator=g).bfloat16()


def gathered(rows, slot):
    here = (slot >= 0) & (slot < rows.shape[0])
    x = rows.double()[torch.where(here, slot, 0).long()]
    return torch.where(here[:, :, None], x, torch.tensor(0.0, dtype=torch.float64)), here


SHAPES = [(1, 16, 1), (1, 4096, 8), (3, 48, 2), (9, 256, 8), (33, 272, 6), (100, 1040, 8), (5, 2064, 31), (2000, 512, 8), (40, 64, 100), (4, 8208, 9)]


@pytest.mark.parametrize("T,n,K", SHAPES)
@pytest.mark.parametrize("weighted", [True, False])
def test_combine(T, n, K, weighted):
    rows, slot, w, _ = case(T, n, K)
    out = Guarded((T, n), torch.bfloat16, fill=9.0, canary=-3.0)
    eqb.eqb_expert_combine(rows.cuda(), slot.cuda(), w.cuda() if weighted else None, out=out.view)
    torch.cuda.synchronize()
    assert out.intact()
    x, _ = gathered(rows, slot)
    ww = w.double()[:, :, None] if weighted else 1.0
    want, mag = (x * ww).sum(1), (x * ww).abs().sum(1)
    assert torch.all((out.view.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + (K + 1) * 2.0 ** -23 * mag)


@pytest.mark.parametrize("T,n,K", SHAPES)
@pytest.mark.parametrize("want", [("rows",), ("weight",), ("rows", "weight")])
@pytest.mark.parametrize("weighted", [True, False])
def test_gradients(T, n, K, want, weighted):
    rows, slot, w, g = case(T, n, K, more=2)
    R = rows.shape[0]
    gr = Guarded((R, n), torch.bfloat16, fill=9.0, canary=-3.0) if "rows" in want else None
    gw = Guarded((T, K), torch.float32, fill=9.0) if "weight" in want else None
    eqb.eqb_expert_combine_grad(g.cuda(), rows.cuda(), slot.cuda(), w.cuda() if weighted else None, grad_rows=gr and gr.view,
                                grad_weight=gw and gw.view)
    torch.cuda.synchronize()
    x, here = gathered(rows, slot)
    if gr:
        assert gr.intact()
        exact = g.float()[:, None, :] * (w if weighted else torch.ones(T, K))[:, :, None]
        full = torch.full((R, n), 9.0).bfloat16()
        full[slot[here].long()] = exact[here].bfloat16()
        assert torch.equal(gr.view.cpu(), full)
    if gw:
        assert gw.intact()
        terms = x * g.double()[:, None, :]
        assert torch.all((gw.view.cpu().double() - terms.sum(2)).abs() <= (n / 32 + 6) * 2.0 ** -24 * terms.abs().sum(2))
        assert not gw.view.cpu()[~here].any()


def test_in_the_place_of_the_rows():
    rows, slot, w, g = case(300, 528, 6)
    apart, gw = eqb.eqb_expert_combine_grad(g.cuda(), rows.cuda(), slot.cuda(), w.cuda(), grad_rows=rows.cuda(),
                                            grad_weight=torch.empty(300, 6, device="cuda"))
    r = rows.cuda()
    same, gw2 = eqb.eqb_expert_combine_grad(g.cuda(), r, slot.cuda(), w.cuda(), grad_rows=r, grad_weight=torch.empty(300, 6, device="cuda"))
    assert torch.equal(gw, gw2) and torch.equal(apart.view(torch.int16), same.view(torch.int16))


def test_slots_that_are_no_rows():
    rows = torch.ones(5, 32, dtype=torch.bfloat16, device="cuda")
    slot = torch.tensor([[0, 5], [-1, -2 ** 31], [2 ** 31 - 1, 4]], dtype=torch.int32, device="cuda")
    out = eqb.eqb_expert_combine(rows, slot)
    assert out[:, 0].tolist() == [1.0, 0.0, 1.0]
    gr = torch.zeros_like(rows)
    _, gw = eqb.eqb_expert_combine_grad(out, rows, slot, grad_rows=gr, grad_weight=torch.empty(3, 2, device="cuda"))
    assert gr[:, 0].tolist() == [1.0, 0.0, 0.0, 0.0, 1.0] and gw.tolist() == [[32.0, 0.0], [0.0, 0.0], [0.0, 32.0]]


def test_differences():
    """The sum is linear in rows and weights: <g, out(x + v) - out(x)> is <grad, v>, exactly on whole numbers."""
    T, n, K = 40, 64, 4
    g0 = torch.Generator().manual_seed(1)
    _, slot, _, _ = case(T, n, K)
    whole = lambda *s: torch.randint(-3, 4, s, generator=g0).float()  # noqa: E731
    rows, w, g, v, u = whole(T * K, n), whole(T, K), whole(T, n), whole(T * K, n), whole(T, K)
    gr = torch.zeros(T * K, n, dtype=torch.bfloat16, device="cuda")
    _, gw = eqb.eqb_expert_combine_grad(g.bfloat16().cuda(), rows.bfloat16().cuda(), slot.cuda(), w.cuda(), grad_rows=gr,
                                        grad_weight=torch.empty(T, K, device="cuda"))
    loss = lambda r, ww: ((gathered(r, slot)[0] * ww.double()[:, :, None]).sum(1) * g.double()).sum()  # noqa: E731
    assert loss(rows + v, w) - loss(rows, w) == (gr.cpu().double() * v.double()).sum()
    assert loss(rows, w + u) - loss(rows, w) == (gw.cpu().double() * u.double()).sum()


def test_nothing_to_do():
    rows = torch.empty(0, 32, dtype=torch.bfloat16, device="cuda")
    out = eqb.eqb_expert_combine(rows, torch.zeros(3, 2, dtype=torch.int32, device="cuda"))
    assert out.shape == (3, 32) and not out.any()
    out = eqb.eqb_expert_combine(rows, torch.zeros(0, 2, dtype=torch.int32, device="cuda"))
    assert out.shape == (0, 32)
