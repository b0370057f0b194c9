"""The experts' operators where element offsets pass 32 bits: the far ends against
plain forms of the same rows."""
import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def filled(T, d, top=3):
    x = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    for a in range(0, T, 1 << 16):
        x[a:a + (1 << 16)] = torch.randint(-top, top + 1, (min(T - a, 1 << 16), d), device="cuda", dtype=torch.int8).bfloat16()
    return x


def test_gate_and_its_gradient():
    T, E, K = 9_000_001, 256, 8
    z = torch.empty(T, E, dtype=torch.bfloat16, device="cuda")
    for a in range(0, T, 1 << 20):
        z[a:a + (1 << 20)] = torch.randn(min(T - a, 1 << 20), E, device="cuda").bfloat16()
    b = torch.randn(E, device="cuda")
    idx, w = eqb.eqb_gate_topk(z, b, K, groups=8, top_groups=4)
    tail = slice(T - 500, T)
    want = ref.choose(z[tail].cpu(), b.cpu(), K, 8, 4)
    assert torch.equal(idx[tail].cpu(), want)
    exact = ref.shares(z[tail].cpu(), want, "sigmoid", True, 1.0)
    assert torch.all((w[tail].cpu().double() - exact).abs() <= 2e-5 * exact)
    gw = torch.randn(T, K, device="cuda")
    dz = eqb.eqb_gate_grad(z, idx, gw, score="softmax", renorm=False)
    full, size = ref.gate_grad(z[tail].cpu(), want, gw[tail].cpu(), "softmax", False, 1.0)
    assert torch.all((dz[tail].cpu().double() - full).abs() <= 2e-5 * size + 1e-30)


def test_rows_quantised_multiplied_and_combined():
    """600,000 rows of 4,096: 2.5 G elements of x, q and rows; whole numbers, so exact."""
    R, d, n, E = 600_000, 4096, 64, 3
    x = filled(R, d, 2)
    x[:, ::128] = 3.5  # the largest of every block: scale 2^-7, and whole numbers are codes
    q, s = eqb.eqb_quant_rows(x)
    assert torch.all(s == 2.0 ** -7)
    off = torch.tensor([0, 7, 599_000, R], dtype=torch.int32, device="cuda")
    w = torch.randint(-1, 2, (E, n, d), device="cuda").float().to(E4M3)
    ws = torch.ones(E, 1, d // 128, device="cuda")
    out = eqb.eqb_expert_matmul(q, s, w, ws, off, out=torch.empty(R, n, device="cuda"))
    for rows, e in ((slice(0, 7), 0), (slice(598_000, 599_000), 1), (slice(R - 1000, R), 2)):
        assert torch.equal(out[rows], (x[rows].double() @ w[e].double().t()).float())
    # the same rows, by token: out and gradients of 2.5 G elements
    slot = torch.arange(R, dtype=torch.int32, device="cuda").flip(0).view(-1, 2).contiguous()
    y = eqb.eqb_expert_combine(x, slot)
    for t in (slice(0, 200), slice(R // 2 - 200, R // 2)):
        assert torch.equal(y[t], x[slot[t].long()].float().sum(1).bfloat16())
    del q, out
    back = torch.empty_like(x)
    _, dw = eqb.eqb_expert_combine_grad(y, x, slot, grad_rows=back, grad_weight=torch.empty(R // 2, 2, device="cuda"))
    for t in (slice(0, 200), slice(R // 2 - 200, R // 2)):
        at = slot[t].long()
        assert torch.equal(back[at], y[t][:, None].expand(-1, 2, -1))
        terms = y[t][:, None].double() * x[at].double()
        assert torch.all((dw[t].double() - terms.sum(2)).abs() <= 200 * 2.0 ** -24 * terms.abs().sum(2))


def test_columns_and_the_weights_gradient():
    """4,096 columns of 5,000 blocks: 2.6 G codes."""
    R, c, E = 640_000, 4096, 2
    off = torch.tensor([0, 300, R], dtype=torch.int32, device="cuda")
    blk = torch.tensor([0, 3, 3 + (R - 300 + 127) // 128], dtype=torch.int32, device="cuda")
    x = filled(R, c, 2)
    x[::64] = 3.5
    q, s = eqb.eqb_quant_cols(x, off, blk)
    last = int(blk[2]) - 1
    rows = x[300 + (last - 3) * 128:]
    wq, wsc = ref.codes(rows.cpu().float(), (0,))
    assert torch.equal(s[last].cpu(), wsc[0])
    assert torch.equal(q[:, last * 128:last * 128 + len(rows)].cpu().view(torch.uint8), wq.t().contiguous().view(torch.uint8))
    # expert 0's 300 rows and expert 1's last blocks as an expert of their own
    tail = torch.tensor([0, 3, 3, last - 4, last + 1], dtype=torch.int32, device="cuda")
    a, sa = q[:32].contiguous(), s[:, :32].contiguous()
    dW = eqb.eqb_expert_wgrad(a, sa, q, s, tail)
    value = lambda rows, at: q[rows, at].double() * s[at.start // 128:at.stop // 128, rows].double().t().repeat_interleave(128, 1)  # noqa: E731
    for e, at in ((0, slice(0, 384)), (3, slice((last - 4) * 128, (last + 1) * 128))):
        u, v = value(slice(0, 32), at), value(slice(0, c), at)
        assert torch.all((dW[e].double() - u @ v.t()).abs() <= 300 * 2.0 ** -24 * (u.abs() @ v.abs().t()))
    assert not dW[1].any()


def test_rows_of_many_lists():
    T, K, E = 4_000_000, 8, 1000
    idx = torch.randint(0, E, (T, K), dtype=torch.int32, device="cuda")
    off, blk, slot, entry = eqb.eqb_expert_rows(idx, E)
    n = torch.bincount(idx.flatten().long(), minlength=E)
    assert torch.equal(off[1:].long(), n.cumsum(0)) and torch.equal(blk[1:].long(), ((n + 127) // 128).cumsum(0))
    order = torch.sort(idx.flatten(), stable=True).indices
    assert torch.equal(entry.long(), order)
    assert torch.equal(slot.flatten()[order].long(), torch.arange(T * K, device="cuda"))
