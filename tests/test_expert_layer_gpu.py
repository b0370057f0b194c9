"""The experts' operators together, as a layer uses them, against autograd in 64 bits:
y_t = sum over t's list of w_tk W_e x_t with the weights from the logits, its gradients
with respect to x, W and the logits.

Each operand of a product is off by at most half a step of e4m3 (2^-4 of it, and
2^-10 of its block's scale), so a sum of products is off by (2 * 2^-4 + 2^-8) of the sum of
their magnitudes and, for the values below the least normal code, of the blocks'
largest magnitudes times 2^-10 / 448, which the factor 1.02 covers at these inputs;
every bf16 result by 2^-8, fp32 sums by far less."""
import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu

PAIR = (2 * 2.0 ** -4 + 2.0 ** -8) * 1.02  # both operands of a product in 8 bits


class Layer:
    """One matrix an expert; what a training step keeps between forward and backward."""

    def __init__(self, W, K, groups=1, top_groups=1, score="sigmoid", scale=2.5):
        self.W, self.K, self.E = W, K, W.shape[0]
        self.gate = {"score": score, "scale": scale, "renorm": True}
        self.groups = {"groups": groups, "top_groups": top_groups, "group_score": "top2"}
        self.q, self.s, self.qt, self.st = eqb.eqb_quant_blocks(W, turned=True)

    def forward(self, x, z, b, mask=None):
        self.x, self.z = x, z
        self.idx, self.w = eqb.eqb_gate_topk(z, b, self.K, mask=mask, **self.gate, **self.groups)
        self.offsets, self.blocks, self.slot, self.entry = eqb.eqb_expert_rows(self.idx, self.E)
        q, s = eqb.eqb_quant_rows(x, self.slot)
        # rows behind the last expert's are left as they are, and no slot names them
        self.rows = eqb.eqb_expert_matmul(q, s, self.q, self.s, self.offsets)
        return eqb.eqb_expert_combine(self.rows, self.slot, self.w)

    def backward(self, dy, dW=None):
        g = torch.empty_like(self.rows)
        _, dw = eqb.eqb_expert_combine_grad(dy, self.rows, self.slot, self.w, grad_rows=g, grad_weight=torch.empty_like(self.w))
        back = torch.empty(self.rows.shape[0], self.x.shape[1], dtype=torch.bfloat16, device="cuda")
        eqb.eqb_expert_matmul(*eqb.eqb_quant_rows(g), self.qt, self.st, self.offsets, out=back)
        dx = eqb.eqb_expert_combine(back, self.slot)
        a, b = eqb.eqb_quant_cols(g, self.offsets, self.blocks), eqb.eqb_quant_cols(self.x, self.offsets, self.blocks, self.entry, self.K)
        dW = eqb.eqb_expert_wgrad(*a, *b, self.blocks, dW=dW, accumulate=dW is not None)
        dz = eqb.eqb_gate_grad(self.z, self.idx, dw, **self.gate)
        return dx, dW, dz, dw


def inputs(T, d, n, E, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    W = torch.randn(E, n, d, generator=g, device="cuda") * d ** -0.5
    z = torch.randn(T, E, generator=g, device="cuda").bfloat16()
    b = torch.randn(E, generator=g, device="cuda") * 0.2
    return x, W, z, b, torch.randn(T, n, generator=g, device="cuda").bfloat16()


def expected(layer, x, W, z, dy):
    """y, dx, dW, dz, dw of the layer's lists by autograd in 64 bits, and the magnitudes that bound their errors."""
    idx = layer.idx.long()
    here, at = idx >= 0, idx.clamp(min=0)
    xd, Wd, zd = (t.double().clone().requires_grad_() for t in (x, W, z))
    zk = torch.where(here, zd.gather(1, at), -torch.inf)
    l = torch.nn.functional.logsigmoid(zk) if layer.gate["score"] == "sigmoid" else zk
    w = torch.where(here, torch.softmax(torch.where(here.any(1, keepdim=True), l, 0.0), 1), 0.0) * layer.gate["scale"]
    w.retain_grad()
    rows = torch.einsum("tkd,tknd->tkn", xd[:, None].expand(-1, layer.K, -1), Wd[at])
    y = (w[:, :, None] * rows).sum(1)
    (y * dy.double()).sum().backward()
    with torch.no_grad():
        mag = torch.einsum("td,tknd->tkn", x.double().abs(), W.double().abs()[at])
        wa, ga = w.detach().abs(), dy.double().abs()
        y_mag = (wa[:, :, None] * mag).sum(1)
        dw_mag = (mag * ga[:, None]).sum(2)
        dx_mag = (wa[:, :, None] * torch.einsum("tn,tknd->tkd", ga, W.double().abs()[at])).sum(1)
        dW_mag = torch.zeros_like(Wd)
        for k in range(layer.K):
            dW_mag.index_add_(0, at[:, k], (wa[:, k] * here[:, k])[:, None, None] * ga[:, :, None] * x.double().abs()[:, None])
    return (y.detach(), xd.grad, Wd.grad, zd.grad, torch.where(here, w.grad, 0.0)), (y_mag, dx_mag, dW_mag, dw_mag)


def check(layer, got, want, mag):
    y, dx, dW, dz, dw = got
    y0, dx0, dW0, dz0, dw0 = want
    y_mag, dx_mag, dW_mag, dw_mag = mag
    half = 2.0 ** -8
    assert torch.all((y.double() - y0).abs() <= (PAIR + 2 * half) * y_mag + half * y0.abs())
    assert torch.all((dw.double() - dw0).abs() <= (PAIR + 2 * half) * dw_mag)
    assert torch.all((dx.double() - dx0).abs() <= (PAIR + 3 * half) * dx_mag + half * dx0.abs())
    assert torch.all((dW.double() - dW0).abs() <= (PAIR + 2 * half) * dW_mag)
    # dz is linear in dw: its formula on the largest errors of dw, and its own rounding
    z, idx = layer.z.cpu(), layer.idx.cpu()
    _, size = ref.gate_grad(z, idx, ((PAIR + 2 * half) * dw_mag).cpu(), **layer.gate)
    _, own = ref.gate_grad(z, idx, dw0.cpu(), **layer.gate)
    assert torch.all((dz.cpu().double() - dz0.cpu()).abs() <= size * 1.01 + 1e-5 * own + 1e-30)


@pytest.mark.parametrize("T,d,n,E,K,groups,score", [(300, 256, 192, 16, 2, 1, "sigmoid"), (700, 400, 144, 32, 4, 4, "softmax"),
                                                     (1, 128, 128, 64, 8, 8, "sigmoid"), (50, 144, 272, 8, 7, 1, "softmax")])
def test_forward_and_backward(T, d, n, E, K, groups, score):
    x, W, z, b, dy = inputs(T, d, n, E, T)
    layer = Layer(W, K, groups, max(1, groups // 2), score)
    y = layer.forward(x, z, b)
    dx, dW, dz, dw = layer.backward(dy)
    want, mag = expected(layer, x, W, z, dy)
    check(layer, (y, dx, dW, dz, dw), want, mag)


def test_a_padded_batch_and_two_microbatches():
    """Padding tokens have no rows and zero outputs; the second microbatch's dW is added to the first's."""
    x, W, z, b, dy = inputs(400, 256, 128, 16, 5)
    mask = torch.arange(400, device="cuda") % 3 != 0
    x[~mask], z[~mask] = torch.nan, torch.nan
    layer = Layer(W, 4)
    total, want_total = None, torch.zeros_like(W, dtype=torch.float64)
    for _ in range(2):
        y = layer.forward(x, z, b, mask=mask)
        dx, total, dz, dw = layer.backward(dy, total)
        assert (layer.idx[~mask] == -1).all() and not y[~mask].any() and not dx[~mask].any() and not dz[~mask].any() and not dw[~mask].any()
        assert torch.isfinite(y).all() and torch.isfinite(dx).all() and torch.isfinite(total).all()
        xc, zc = torch.where(mask[:, None], x, 0), torch.where(mask[:, None], z, 0)
        want, mag = expected(layer, xc, W, zc, dy)
        want_total += want[2]
        assert torch.all((y.double() - want[0]).abs() <= (PAIR + 2.0 ** -7) * mag[0] + 2.0 ** -8 * want[0].abs())
    assert torch.all((total.double() - want_total).abs() <= 2 * (PAIR + 2.0 ** -7) * mag[2])


def test_into_the_router_and_its_balance():
    """dz goes on into the balance loss and the projection's gradients, in the types that those take."""
    T, d, E, K = 256, 128, 16, 2
    x, W, _, b, dy = inputs(T, d, 64, E, 6)
    Wr = (torch.randn(E, d, device="cuda") * d ** -0.5).bfloat16()
    z = eqb.eqb_router_logits(x, Wr)
    layer = Layer(W, K)
    layer.forward(x, z, b)
    dz = layer.backward(dy)[2]
    off = torch.tensor([0, T], device="cuda")
    both = torch.empty(T, E, dtype=torch.bfloat16, device="cuda")
    eqb.eqb_balance_loss(z, layer.idx, off, 0.01, score="sigmoid", grad_in=dz, grad_out=both)
    dWr = torch.empty(E, d, device="cuda")
    eqb.eqb_router_grad(both, x, Wr, dW=dWr)
    want = both.double().t() @ x.double()
    assert torch.all((dWr.double() - want).abs() <= 1e-5 * (both.double().abs().t() @ x.double().abs()))
    assert (both.float() - dz).abs().max() > 0  # the balance loss is in it


def test_in_a_graph():
    """Forward and backward captured and replayed on other inputs, twice, while another layer's runs eagerly."""
    x, W, z, b, dy = inputs(900, 256, 256, 32, 7)
    layer, other = Layer(W, 4, 4, 2), Layer(W, 4, 4, 2)

    def step(at):
        y = at.forward(x, z, b)
        return (y,) + at.backward(dy)

    step(layer)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(layer)
    for seed in (8, 9):
        new = inputs(900, 256, 256, 32, seed)
        x.copy_(new[0])
        z.copy_(new[2])
        dy.copy_(new[4])
        graph.replay()
        want = step(other)
        for g, w in zip(got, want):
            assert torch.equal(g, w)
