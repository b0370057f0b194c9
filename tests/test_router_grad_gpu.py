"""eqb_router_grad: exact on whole numbers, and against 64 bits on others.

dW accumulates in fp32 on the tensor cores, 16 tokens at a time: at most
(T / 16 + 24) roundings of 2^-23 of the sum of the products' magnitudes (24 for
the parts and what the output held).  dx sums at most 256 products: 40 such
roundings, then one to bf16 (2^-8)."""
import numpy as np
import pytest
import torch

import paper_2609_28053_gb300 as eqb
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu


def run(dz, x, W, add_dx=False, add_dW=False, dx0=None, dW0=None, want=("dx", "dW")):
    T, E = dz.shape
    d = x.shape[1]
    dx = Guarded((T, d), torch.bfloat16, fill=5.0, canary=-3.0) if "dx" in want else None
    dW = Guarded((E, d), torch.float32, fill=5.0) if "dW" in want else None
    if dx is not None and dx0 is not None:
        dx.view.copy_(dx0)
    if dW is not None and dW0 is not None:
        dW.view.copy_(dW0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.full((max(1, eqb.eqb_router_grad_workspace_bytes(T, d, E)),), 0xff, dtype=torch.uint8, device="cuda")
    eqb.eqb_router_grad(dz.cuda(), x.cuda(), W.cuda(), dx=dx and dx.view, dW=dW and dW.view, accumulate_dx=add_dx,
                        accumulate_dW=add_dW, workspace=ws, err_flag=err)
    torch.cuda.synchronize()
    assert err.item() == 0
    for b in (dx, dW):
        assert b is None or b.intact()
    return dx and dx.view.cpu(), dW and dW.view.cpu()


def whole(T, d, E, seed):
    """Small whole numbers: every sum is exact in fp32 (below 2^24)."""
    g = torch.Generator().manual_seed(seed)
    dz = torch.randint(-2, 3, (T, E), generator=g).bfloat16()
    x = torch.randint(-3, 4, (T, d), generator=g).bfloat16()
    W = torch.randint(-2, 3, (E, d), generator=g).bfloat16()
    return dz, x, W


SHAPES = [(1, 64, 16), (2, 64, 48), (63, 128, 64), (64, 192, 16), (65, 320, 96), (127, 64, 128), (129, 1024, 144),
          (300, 1024, 64), (300, 448, 256), (1000, 256, 240), (1000, 2048, 128), (2500, 704, 256), (5000, 64, 32),
          (40000, 128, 16), (20000, 256, 256)]


@pytest.mark.parametrize("T,d,E", SHAPES)
def test_exact_on_whole_numbers(T, d, E):
    dz, x, W = whole(T, d, E, T + d + E)
    dx, dW = run(dz, x, W)
    assert torch.equal(dx, (dz.float() @ W.float()).bfloat16())
    assert torch.equal(dW, (dz.double().t() @ x.double()).float())


@pytest.mark.parametrize("T,d,E", [(1, 64, 16), (300, 448, 256), (1000, 2048, 128), (2500, 704, 48), (20000, 256, 256)])
def test_accumulates(T, d, E):
    dz, x, W = whole(T, d, E, T)
    g = torch.Generator().manual_seed(1)
    dx0 = torch.randint(-60, 60, (T, d), generator=g).bfloat16()
    dW0 = torch.randint(-1000, 1000, (E, d), generator=g).float()
    dx, dW = run(dz, x, W, True, True, dx0, dW0)
    assert torch.equal(dx, (dz.float() @ W.float() + dx0.float()).bfloat16())
    assert torch.equal(dW, (dz.double().t() @ x.double() + dW0.double()).float())
    dx, dW = run(dz, x, W, True, False, dx0, dW0)
    assert torch.equal(dx, (dz.float() @ W.float() + dx0.float()).bfloat16())
    assert torch.equal(dW, (dz.double().t() @ x.double()).float())


def test_one_output():
    dz, x, W = whole(700, 256, 64, 3)
    dx, none = run(dz, x, W, want=("dx",))
    assert none is None and torch.equal(dx, (dz.float() @ W.float()).bfloat16())
    none, dW = run(dz, x, W, want=("dW",))
    assert none is None and torch.equal(dW, dz.float().t() @ x.float())


@pytest.mark.parametrize("T,d,E", [(333, 512, 64), (4100, 1024, 256), (70000, 256, 128)])
def test_against_64_bits(T, d, E):
    g = torch.Generator(device="cuda").manual_seed(T)
    dz = torch.randn(T, E, generator=g, device="cuda").bfloat16()
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    W = torch.randn(E, d, generator=g, device="cuda").bfloat16()
    dx, dW = run(dz, x, W)
    zd, xd, wd = dz.double(), x.double(), W.double()
    want, size = (zd.t() @ xd).cpu(), (zd.abs().t() @ xd.abs()).cpu()
    assert torch.all((dW.double() - want).abs() <= (T / 16 + 24) * 2.0 ** -23 * size)
    want, size = (zd @ wd).cpu(), (zd.abs() @ wd.abs()).cpu()
    assert torch.all((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + 40 * 2.0 ** -23 * size)


def test_against_differences():
    """z is linear: <dz, z(x + s) - z(x)> = <dx, s> and the same for W_r, exactly on whole numbers."""
    T, d, E = 130, 128, 32
    dz, x, W = whole(T, d, E, 5)
    dx, dW = run(dz, x, W)
    s = torch.zeros(T, d, dtype=torch.float64)
    s[::7, ::5] = 1.0
    z = lambda a, b: (dz.double() * (a.double() @ b.double().t())).sum()  # noqa: E731
    exact_dx = dz.double() @ W.double()
    assert z(x.double() + s, W) - z(x, W) == (exact_dx * s).sum()
    assert torch.equal(dx, exact_dx.bfloat16())
    s = torch.zeros(E, d, dtype=torch.float64)
    s[::3, ::4] = 1.0
    assert z(x, W.double() + s) - z(x, W) == (dW.double() * s).sum()


def test_no_tokens():
    z = torch.empty(0, 64, dtype=torch.bfloat16)
    x = torch.empty(0, 128, dtype=torch.bfloat16)
    W = torch.ones(64, 128, dtype=torch.bfloat16)
    dx, dW = run(z, x, W)
    assert dx.shape == (0, 128) and not dW.any()
    dW0 = torch.randn(64, 128)
    assert torch.equal(run(z, x, W, add_dW=True, dW0=dW0)[1], dW0)


def test_same_bits():
    g = torch.Generator(device="cuda").manual_seed(2)
    dz = torch.randn(9000, 128, generator=g, device="cuda").bfloat16()
    x = torch.randn(9000, 512, generator=g, device="cuda").bfloat16()
    W = torch.randn(128, 512, generator=g, device="cuda").bfloat16()
    a, b = run(dz, x, W), run(dz, x, W)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
