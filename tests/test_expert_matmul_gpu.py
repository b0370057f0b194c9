"""eqb_expert_matmul and eqb_expert_wgrad: exact on whole numbers, and against 64
bits on others.

A block's 128 products are exact; the tensor cores add 32 of them to a sum at a time
and cut off what is below the last of 24 places of the largest term: at most 33 cuts
a step, 4 steps, of 2^-23 of the block's sum of magnitudes.  The scales' product is
one rounding, and the sum over the blocks one a block: (132 * 2 + blocks + 2) 2^-24 of
the sum of all magnitudes; then one rounding to bf16 (2^-8)."""
import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def up(n):
    return (n + 127) // 128


def offsets_of(lens):
    return torch.tensor([0] + lens, dtype=torch.int32).cumsum(0).int()


def codes(shape, g, top=None):
    if top is not None:  # whole numbers
        return torch.randint(-top, top + 1, shape, generator=g, device="cuda").float().to(E4M3)
    return (torch.randn(shape, generator=g, device="cuda") * 100).clamp(-448, 448).to(E4M3)


def powers(shape, g):
    return torch.exp2(torch.randint(-2, 3, shape, generator=g, device="cuda").float())


def run(q, s, w, ws, offsets, fp32=False):
    R, n = q.shape[0], w.shape[1]
    out = Guarded((R, n), torch.float32 if fp32 else torch.bfloat16, fill=-5.0, canary=-3.0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    eqb.eqb_expert_matmul(q, s, w, ws, offsets.cuda(), out=out.view, err_flag=err)
    torch.cuda.synchronize()
    assert err.item() == 0 and out.intact()
    return out.view


def product(q, s, w, ws, offsets):
    """In 64 bits, with the sum of magnitudes."""
    R, d = q.shape
    E, n, _ = w.shape
    out, mag = torch.zeros(R, n, dtype=torch.float64, device="cuda"), torch.zeros(R, n, dtype=torch.float64, device="cuda")
    for e in range(E):
        a, b = int(offsets[e]), int(offsets[e + 1])
        if a < b:
            x = q[a:b].double() * ref.spread(s[a:b].double(), 1, d)
            y = w[e].double() * ref.spread(ref.spread(ws[e].double(), 0, n), 1, d)
            out[a:b], mag[a:b] = x @ y.t(), x.abs() @ y.abs().t()
    return out, mag


SHAPES = [([1], 16, 16), ([1], 64, 128), ([0, 0, 1, 0], 48, 64), ([3, 0, 5], 256, 144), ([31, 32, 33, 64, 65], 272, 256), ([96, 97, 127], 128, 400),
          ([128], 256, 512), ([129, 1, 255], 512, 128), ([300, 0, 7, 500], 528, 1040), ([2000, 3000], 1024, 256), ([0] * 40, 64, 64),
          ([1] * 300, 320, 272), ([700] * 30, 256, 512), ([5, 0, 260] * 40, 1296, 128)]


@pytest.mark.parametrize("lens,n,d", SHAPES)
def test_exact_on_whole_numbers(lens, n, d):
    """Codes of whole numbers and scales of powers of two: every sum is exact (below 2^24 steps of 2^-4)."""
    g = torch.Generator(device="cuda").manual_seed(n + d + len(lens))
    R, E = sum(lens) + 3, len(lens)
    q, w = codes((R, d), g, 4), codes((E, n, d), g, 3)
    s, ws = powers((R, up(d)), g), powers((E, up(n), up(d)), g)
    off = offsets_of(lens)
    want, _ = product(q, s, w, ws, off)
    got = run(q, s, w, ws, off, fp32=True)
    assert torch.equal(got[:-3], want[:-3].float()) and (got[-3:] == -5.0).all()  # behind the last row: as it was
    got = run(q, s, w, ws, off)
    assert torch.equal(got[:-3], want[:-3].float().bfloat16()) and (got[-3:] == -5.0).all()


@pytest.mark.parametrize("lens,n,d", [([7, 120, 0, 33], 272, 1040), ([500, 300], 512, 2048), ([3] * 20, 64, 528), ([2000] * 12, 768, 512)])
@pytest.mark.parametrize("fp32", [False, True])
def test_against_64_bits(lens, n, d, fp32):
    g = torch.Generator(device="cuda").manual_seed(n)
    R, E = sum(lens), len(lens)
    q, w = codes((R, d), g), codes((E, n, d), g)
    s = torch.exp(torch.randn((R, up(d)), generator=g, device="cuda"))
    ws = torch.exp(torch.randn((E, up(n), up(d)), generator=g, device="cuda"))
    off = offsets_of(lens)
    want, mag = product(q, s, w, ws, off)
    got = run(q, s, w, ws, off, fp32).double()
    tol = (132 * 2 + up(d) + 2) * 2.0 ** -24 * mag
    if not fp32:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    assert torch.all((got - want).abs() <= tol)


def test_rows_do_not_touch_each_other():
    """A NaN code stays in its row, and rows of no expert in none."""
    g = torch.Generator(device="cuda").manual_seed(5)
    q, w = codes((200, 256), g, 4), codes((2, 64, 256), g, 3)
    s, ws = powers((200, 2), g), powers((2, 1, 2), g)
    q.view(torch.uint8)[50] = 0x7f
    q.view(torch.uint8)[150:] = 0x7f  # behind the last row
    off = offsets_of([60, 90])
    got = run(q, s, w, ws, off, fp32=True)
    q2 = q.clone()
    q2.view(torch.uint8)[50] = 0
    want, _ = product(q2, s, w, ws, off)
    keep = torch.arange(150, device="cuda") != 50
    assert torch.equal(got[:150][keep], want[:150][keep].float()) and torch.isnan(got[50]).all()


def test_offsets_that_lie():
    """Whatever the offsets say, nothing outside the buffers is written."""
    g = torch.Generator(device="cuda").manual_seed(6)
    q, w = codes((100, 128), g, 4), codes((3, 64, 128), g, 3)
    s, ws = powers((100, 1), g), powers((3, 1, 1), g)
    for off in ([0, 50, 40, 100], [0, 2 ** 30, 100, 100], [-7, -3, 20, 2000], [90, 10, 10, 10]):
        run(q, s, w, ws, torch.tensor(off, dtype=torch.int32))


def test_the_gradient_of_the_input_is_the_product_with_the_turned_weights():
    g = torch.Generator(device="cuda").manual_seed(7)
    lens, n, d = [90, 0, 200], 272, 144
    off = offsets_of(lens)
    w = torch.randint(-3, 4, (3, n, d), generator=g, device="cuda").float()
    w[:, 0, :] = 448.0  # with 448 in every block of 128 x 128 and of its transpose the codes are the values
    w[:, 128::128, :], w[:, :, ::128] = 448.0, 448.0
    wq, ws, wt, wts = eqb.eqb_quant_blocks(w, turned=True)
    assert (ws == 1.0).all()
    dy = codes((290, n), g, 2)
    got = run(dy, torch.ones(290, up(n), device="cuda"), wt, wts, off, fp32=True)
    want = torch.cat([dy[:90].double() @ w[0].double(), dy[90:].double() @ w[2].double()])
    assert torch.equal(got, want.float())


# ---- the gradient of the weights

def run_wgrad(a, sa, b, sb, blocks, add=False, dW0=None):
    E, n, d = blocks.numel() - 1, a.shape[0], b.shape[0]
    dW = Guarded((E, n, d), torch.float32, fill=7.0)
    if dW0 is not None:
        dW.view.copy_(dW0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    eqb.eqb_expert_wgrad(a, sa, b, sb, blocks.cuda(), dW=dW.view, accumulate=add, err_flag=err)
    torch.cuda.synchronize()
    assert err.item() == 0 and dW.intact()
    return dW.view


def wgrad(a, sa, b, sb, blocks):
    E, n, d = blocks.numel() - 1, a.shape[0], b.shape[0]
    out, mag = torch.zeros(E, n, d, dtype=torch.float64, device="cuda"), torch.zeros(E, n, d, dtype=torch.float64, device="cuda")
    for e in range(E):
        for k in range(int(blocks[e]), int(blocks[e + 1])):
            x = a[:, k * 128:(k + 1) * 128].double() * sa[k].double()[:, None]
            y = b[:, k * 128:(k + 1) * 128].double() * sb[k].double()[:, None]
            out[e] += x @ y.t()
            mag[e] += x.abs() @ y.abs().t()
    return out, mag


@pytest.mark.parametrize("blk,n,d", [([1], 16, 16), ([1], 128, 256), ([0, 2, 0], 144, 272), ([3, 1, 4], 256, 512), ([0, 0], 64, 64),
                                     ([5, 0, 1, 7], 400, 1040), ([2] * 30, 256, 768), ([40], 272, 528)])
@pytest.mark.parametrize("add", [False, True])
def test_wgrad_exact_on_whole_numbers(blk, n, d, add):
    g = torch.Generator(device="cuda").manual_seed(n + d)
    P = max(1, sum(blk) + 1)
    a, b = codes((n, P * 128), g, 2), codes((d, P * 128), g, 3)
    sa, sb = powers((P, n), g), powers((P, d), g)
    blocks = offsets_of(blk)
    want, _ = wgrad(a, sa, b, sb, blocks)
    dW0 = torch.randint(-50, 50, want.shape, generator=g, device="cuda").float()
    got = run_wgrad(a, sa, b, sb, blocks, add, dW0)
    assert torch.equal(got, (want + dW0.double() if add else want).float())


@pytest.mark.parametrize("E,n,d", [(100, 144, 1040), (1024, 16, 2064), (1000, 16, 1808)])
def test_wgrad_of_many_unlike_experts(E, n, d):
    """Tiles go by the experts' sizes, not by their numbers; equal and empty ones are among them."""
    g = torch.Generator(device="cuda").manual_seed(5)
    blk = [(7 * e) % 5 if e % 3 else 0 for e in range(E)]
    P = sum(blk)
    a, b = codes((n, P * 128), g, 2), codes((d, P * 128), g, 3)
    sa, sb = powers((P, n), g), powers((P, d), g)
    blocks = offsets_of(blk)
    want, _ = wgrad(a, sa, b, sb, blocks)
    assert torch.equal(run_wgrad(a, sa, b, sb, blocks).double(), want)


@pytest.mark.parametrize("blk,n,d", [([3, 0, 9], 272, 144), ([20, 4], 128, 1040)])
def test_wgrad_against_64_bits(blk, n, d):
    g = torch.Generator(device="cuda").manual_seed(n)
    P = sum(blk)
    a, b = codes((n, P * 128), g), codes((d, P * 128), g)
    sa, sb = (torch.exp(torch.randn((P, k), generator=g, device="cuda")) for k in (n, d))
    blocks = offsets_of(blk)
    want, mag = wgrad(a, sa, b, sb, blocks)
    got = run_wgrad(a, sa, b, sb, blocks).double()
    assert torch.all((got - want).abs() <= (132 * 2 + max(blk) + 2) * 2.0 ** -24 * mag)


def test_wgrad_of_no_blocks():
    e = torch.zeros(3, dtype=torch.int32)
    a, b = torch.empty(64, 0, dtype=E4M3, device="cuda"), torch.empty(48, 0, dtype=E4M3, device="cuda")
    s1, s2 = torch.empty(0, 64, device="cuda"), torch.empty(0, 48, device="cuda")
    assert not run_wgrad(a, s1, b, s2, e).any()
    assert (run_wgrad(a, s1, b, s2, e, add=True) == 7.0).all()


def test_blocks_that_lie():
    g = torch.Generator(device="cuda").manual_seed(6)
    a, b = codes((64, 256), g, 2), codes((48, 256), g, 3)
    sa, sb = powers((2, 64), g), powers((2, 48), g)
    for blk in ([0, 50, 2], [-4, 1, 2 ** 30], [2, 1, 0]):
        run_wgrad(a, sa, b, sb, torch.tensor(blk, dtype=torch.int32))


def test_same_bits_and_streams():
    """The same call twice, the second captured on another stream and replayed beside the first's."""
    g = torch.Generator(device="cuda").manual_seed(8)
    q, w = codes((3000, 512), g), codes((8, 640, 512), g)
    s = torch.rand(3000, 4, generator=g, device="cuda")
    ws = torch.rand(8, 5, 4, generator=g, device="cuda")
    off = offsets_of([375] * 8).cuda()
    first = eqb.eqb_expert_matmul(q, s, w, ws, off)
    second = torch.empty_like(first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eqb.eqb_expert_matmul(q, s, w, ws, off, out=second)
        graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        eqb.eqb_expert_matmul(q, s, w, ws, off, out=second)
    second.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.replay()
    third = eqb.eqb_expert_matmul(q, s, w, ws, off)
    torch.cuda.synchronize()
    assert torch.equal(first, second) and torch.equal(first, third)


def test_nothing_to_do():
    w, ws = torch.zeros(2, 64, 32, device="cuda").to(E4M3), torch.zeros(2, 1, 1, device="cuda")
    out = eqb.eqb_expert_matmul(torch.empty(0, 32, dtype=E4M3, device="cuda"), torch.empty(0, 1, device="cuda"), w, ws,
                                torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert out.shape == (0, 64)


def test_refusals():
    w, ws = torch.zeros(2, 64, 32, device="cuda").to(E4M3), torch.zeros(2, 1, 1, device="cuda")
    q, s, off = torch.zeros(4, 32, device="cuda").to(E4M3), torch.zeros(4, 1, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="w_scale"):
        eqb.eqb_expert_matmul(q, s, w, ws[:1], off)
    with pytest.raises(ValueError, match="offsets"):
        eqb.eqb_expert_matmul(q, s, w, ws, off[:2])
    with pytest.raises(TypeError, match="q must be"):
        eqb.eqb_expert_matmul(q.float(), s, w, ws, off)
    out = torch.empty(4 * 64 + 8, dtype=torch.bfloat16, device="cuda")[8:].view(4, 64)  # 16 bytes late
    with pytest.raises(eqb.EqbError, match="INVALID"):
        eqb.eqb_expert_matmul(q, s, w, ws, off, out=out)
    with pytest.raises(ValueError, match="accumulate"):
        eqb.eqb_expert_wgrad(torch.zeros(64, 128, device="cuda").to(E4M3), torch.zeros(1, 64, device="cuda"),
                             torch.zeros(32, 128, device="cuda").to(E4M3), torch.zeros(1, 32, device="cuda"), off, accumulate=True)
