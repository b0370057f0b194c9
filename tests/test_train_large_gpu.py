"""The training operators where element offsets pass 32 bits: the far ends
against plain forms of the same rows."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


def test_balance_loss_past_2_to_31_elements():
    """2.3 G logits; the last microbatch against torch in 64 bits.  Tolerances as
    in the balance loss's own tests, and 2^-8 for the bf16 gradient."""
    T, E, K, M = 9_000_001, 256, 8, 3
    z = torch.empty(T, E, dtype=torch.bfloat16, device="cuda")
    for a in range(0, T, 1 << 20):
        z[a:a + (1 << 20)] = torch.randn(min(T - a, 1 << 20), E, device="cuda").bfloat16()
    idx = torch.randint(0, E, (T, K), dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 5, T - 3001, T], device="cuda")
    out = torch.empty_like(z)
    prob = torch.empty(M, E, device="cuda")
    loss, counts = eqb.eqb_balance_loss(z, idx, off, 0.1, grad_out=out, prob=prob)
    zz = z[-3001:].double()
    want = torch.bincount(idx[-3001:].flatten().long(), minlength=E)
    assert torch.equal(counts[2].long(), want)
    assert torch.equal(counts.sum(0).long(), torch.bincount(idx.flatten().long(), minlength=E))
    p = torch.softmax(zz, 1)
    F = want.double() / (K * 3001)
    g = 0.1 / 3001 * p * (F - (p @ F)[:, None])
    size = 0.1 / 3001 * p * ((F - 1 / E).abs() + ((p @ F) - 1 / E).abs()[:, None] + 1e-6 / E)
    assert torch.all((out[-3001:].double() - g).abs() <= 2e-5 * size + 2.0 ** -8 * g.abs() * 1.01 + 1e-30)
    assert torch.all((prob[2] - p.mean(0)).abs() <= 1e-5 * p.mean(0))


def test_router_grad_past_2_to_31_elements():
    """2.5 G elements of x and dx, whole numbers: exact."""
    T, d, E = 600_000, 4096, 16
    dz = torch.randint(-1, 2, (T, E), device="cuda").bfloat16()
    x = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    for a in range(0, T, 1 << 16):
        x[a:a + (1 << 16)] = torch.randint(-2, 3, (min(T - a, 1 << 16), d), device="cuda", dtype=torch.int8).bfloat16()
    W = torch.randint(-2, 3, (E, d), device="cuda").bfloat16()
    dx, dW = torch.empty_like(x), torch.empty(E, d, device="cuda")
    eqb.eqb_router_grad(dz, x, W, dx=dx, dW=dW)
    want = torch.zeros(E, d, dtype=torch.float64, device="cuda")
    for a in range(0, T, 1 << 16):
        want += dz[a:a + (1 << 16)].double().t() @ x[a:a + (1 << 16)].double()
    assert torch.equal(dW.double(), want)
    for rows in (slice(0, 300), slice(T // 2, T // 2 + 300), slice(T - 300, T)):
        assert torch.equal(dx[rows], (dz[rows].float() @ W.float()).bfloat16())


def test_router_grad_added_past_2_to_31_elements():
    """The same with both gradients added to: whole numbers below 2^8 in bf16 and
    below 2^24 in fp32, so exact."""
    T, d, E = 530_003, 4096, 32
    dz = torch.randint(-1, 2, (T, E), device="cuda").bfloat16()
    x, dx = (torch.empty(T, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (x, dx):
        for a in range(0, T, 1 << 16):
            t[a:a + (1 << 16)] = torch.randint(-2, 3, (min(T - a, 1 << 16), d), device="cuda", dtype=torch.int8).bfloat16()
    W = torch.randint(-2, 3, (E, d), device="cuda").bfloat16()
    dW = torch.randint(-100, 101, (E, d), device="cuda").float()
    places = [slice(0, 300), slice(T // 2, T // 2 + 300), slice(T - 300, T)]
    old, want = [dx[rows].float() for rows in places], dW.double()
    for a in range(0, T, 1 << 16):
        want += dz[a:a + (1 << 16)].double().t() @ x[a:a + (1 << 16)].double()
    eqb.eqb_router_grad(dz, x, W, dx=dx, dW=dW, accumulate_dx=True, accumulate_dW=True)
    assert torch.equal(dW.double(), want)
    for rows, o in zip(places, old):
        assert torch.equal(dx[rows], (o + dz[rows].float() @ W.float()).bfloat16())


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_past_2_to_31_elements(bits):
    """A tensor of 2^31 + 70,000 elements: its last 2^18 as a tensor of their own give the same bits."""
    n, m = (1 << 31) + 70_000 - 176, 1 << 18  # n a multiple of 256 and m of them
    n -= n % 256
    p = torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_(std=0.02)
    g = torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_(std=1e-3)
    ps, gs = p[-m:].clone(), g[-m:].clone()
    big, small = eqb.EqbAdamW([p], state_bits=bits), eqb.EqbAdamW([ps], state_bits=bits)
    for step in (1, 2):
        big.step([g], lr=1e-3, step=step)
        small.step([gs], lr=1e-3, step=step)
    assert torch.equal(p[-m:], ps)
    assert torch.equal(big.exp_avg[0][-m:].float(), small.exp_avg[0].float())
    assert torch.equal(big.exp_avg_sq[0][-m:].float(), small.exp_avg_sq[0].float())
    if bits == 8:
        assert torch.equal(big.sq_scale[0][-m // 256:], small.sq_scale[0])


def test_refusals_of_layouts():
    """Transposed and strided tensors are refused, and wrong shapes."""
    z = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    idx = torch.zeros(64, 4, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 64], device="cuda")
    for bad in (dict(z=z.t()), dict(idx=idx[:, ::2]), dict(grad_out=torch.empty(64, 128, device="cuda")[:, ::2]),
                dict(counts=torch.empty(2, 64, dtype=torch.int32, device="cuda")), dict(prob=torch.empty(64, device="cuda"))):
        kw = dict(grad_out=None, counts=None, prob=None) | {k: v for k, v in bad.items() if k not in ("z", "idx")}
        with pytest.raises(ValueError):
            eqb.eqb_balance_loss(bad.get("z", z), bad.get("idx", idx), off, 0.1, **kw)
    with pytest.raises(ValueError, match="score"):
        eqb.eqb_balance_loss(z, idx, off, 0.1, score="tanh")
    with pytest.raises(TypeError):
        eqb.eqb_balance_loss(z.half(), idx, off, 0.1)
    with pytest.raises(eqb.EqbError):
        eqb.eqb_balance_loss(z, idx, off, 0.1, score="sigmoid", zeta=0.1)
    x = torch.zeros(64, 128, dtype=torch.bfloat16, device="cuda")
    W = torch.zeros(64, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        eqb.eqb_router_grad(z, x.t().contiguous().t(), W, dx=torch.empty_like(x))
    with pytest.raises(TypeError):
        eqb.eqb_router_grad(z.float(), x, W, dx=torch.empty_like(x))
    with pytest.raises(TypeError):
        eqb.eqb_router_grad(z, x, W, dW=torch.empty(64, 128, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(eqb.EqbError):
        eqb.eqb_router_grad(z, x[:, :96].contiguous(), W[:, :96].contiguous(), dx=torch.empty(64, 96, dtype=torch.bfloat16, device="cuda"))
