"""eqb_quant_rows, eqb_quant_cols and eqb_quant_blocks: codes and scales are equal to
the documented operations one by one in fp32, and a value is within half a step
of e4m3 (2^-4 of it, or 2^-10 of the scale where codes are subnormal) and the two
roundings before it (2 * 2^-24) of what it was."""
import math

import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def values(shape, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(2 * torch.randn(shape[:-1] + (1,), generator=g))
    x[..., ::37] *= 50.0
    x.view(-1)[:200] = 0.0
    return x


def guarded8(shape):
    b = Guarded(shape, torch.uint8, fill=0x55, canary=77)
    return b, b.view.view(E4M3)


def raw(t):
    return t.view(torch.uint8)


def near(q, spread_scale, x):
    back = q.double() * spread_scale.double()
    return torch.all((back - x.double()).abs() <= (2.0 ** -4 + 2.0 ** -22) * x.double().abs() + 2.0 ** -10 * spread_scale.double())


def padded(x, *dims):
    for d in dims:
        more = -x.shape[d] % 128
        if more:
            x = torch.cat([x, x.new_zeros([more if i == d % x.dim() else n for i, n in enumerate(x.shape)])], d)
    return x


def want_rows(x):
    T, d = x.shape
    q, s = ref.codes(padded(x.float(), 1).view(T, -1, 128), (2,))
    return q.reshape(T, -1)[:, :d], s[..., 0]


@pytest.mark.parametrize("T,d", [(1, 16), (1, 4096), (3, 128), (5, 144), (7, 496), (9, 512), (33, 528), (64, 1024), (130, 2064), (2, 8192),
                                 (5000, 1040)])
def test_rows(T, d):
    x = values((T, d), T + d).bfloat16()
    b, q = guarded8((T, d))
    s = Guarded((T, (d + 127) // 128), torch.float32)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    eqb.eqb_quant_rows(x.cuda(), q=q, scale=s.view, err_flag=err)
    torch.cuda.synchronize()
    assert b.intact() and s.intact() and err.item() == 0
    wq, ws = want_rows(x)
    assert torch.equal(s.view.cpu(), ws) and torch.equal(raw(q).cpu(), raw(wq.contiguous()))
    assert near(q.cpu(), ref.spread(s.view.cpu(), 1, d), x)


@pytest.mark.parametrize("T,d,E,K", [(1, 64, 8, 2), (1, 64, 64, 40), (17, 144, 8, 2), (200, 1024, 16, 8), (3000, 272, 64, 6)])
@pytest.mark.parametrize("drop", [0.0, 0.4])
def test_rows_to_slots(T, d, E, K, drop):
    g = torch.Generator().manual_seed(T)
    x = values((T, d), T).bfloat16()
    idx = torch.randint(0, E, (T, K), generator=g, dtype=torch.int32)
    idx[torch.rand(T, K, generator=g) < drop] = -1
    if drop:
        idx[0] = -1
        x[0] = math.nan  # goes nowhere and is not looked at
    _, _, slot, entry = ref.rows(idx, E)
    b, q = guarded8((T * K, d))
    s = Guarded((T * K, (d + 127) // 128), torch.float32, fill=-3.0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    eqb.eqb_quant_rows(x.cuda(), slot=torch.tensor(slot, dtype=torch.int32, device="cuda").view(T, K), q=q, scale=s.view, err_flag=err)
    torch.cuda.synchronize()
    assert b.intact() and s.intact() and err.item() == 0
    wq, ws = want_rows(x)
    token = torch.tensor(entry).div(K, rounding_mode="floor")
    have = torch.tensor(entry) >= 0
    assert torch.equal(s.view.cpu()[have], ws[token[have]]) and torch.equal(raw(q).cpu()[have], raw(wq.contiguous())[token[have]])
    assert (s.view.cpu()[~have] == -3.0).all() and (raw(q).cpu()[~have] == 0x55).all()  # left as they were


def test_slots_that_are_no_rows_are_left_out():
    x = values((4, 64), 1).bfloat16()
    slot = torch.tensor([[0, 8], [-1, 7], [-2 ** 31, 2 ** 31 - 1], [3, 100]], dtype=torch.int32)
    b, q = guarded8((8, 64))
    s = Guarded((8, 1), torch.float32, fill=-3.0)
    eqb.eqb_quant_rows(x.cuda(), slot=slot.cuda(), q=q, scale=s.view)
    torch.cuda.synchronize()
    assert b.intact() and s.intact()
    wq, _ = want_rows(x)
    for r, t in ((0, 0), (7, 1), (3, 3)):
        assert torch.equal(raw(q).cpu()[r], raw(wq.contiguous())[t])
    assert (s.view.cpu()[[1, 2, 4, 5, 6]] == -3.0).all()


@pytest.mark.parametrize("at", [0, 130, 255])
@pytest.mark.parametrize("bad", [math.nan, -math.nan, math.inf, -math.inf])
def test_nonfinite_raises_the_flag_for_its_block_alone(bad, at):
    x = values((6, 256), 2)
    x[3, at] = bad
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    q, s = eqb.eqb_quant_rows(x.bfloat16().cuda(), err_flag=err)
    assert err.item() == 4
    wq, ws = want_rows(x.bfloat16())
    ok = torch.ones(6, 2, dtype=torch.bool)
    ok[3, at // 128] = False
    assert torch.equal(s.cpu()[ok], ws[ok])
    assert torch.equal(raw(q).cpu().view(6, 2, 128)[ok], raw(wq.contiguous()).view(6, 2, 128)[ok])
    for w in (x.view(1, 96, 16), x.bfloat16().view(1, 96, 16)):
        err.zero_()
        eqb.eqb_quant_blocks(w.cuda(), err_flag=err)
        assert err.item() == 4
    err.zero_()
    off = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    eqb.eqb_quant_cols(x.bfloat16().cuda(), off, off.clamp(max=1), err_flag=err)
    assert err.item() == 4


@pytest.mark.parametrize("top", [3.3e38, 1e-30, 2.0 ** -118, 2.0 ** -117, 1e-38, 2.0 ** -133])
def test_the_ends_of_the_range(top):
    x = torch.linspace(-1, 1, 256).view(2, 128) * top
    q, s = eqb.eqb_quant_rows(x.bfloat16().cuda())
    wq, ws = want_rows(x.bfloat16())
    assert torch.equal(s.cpu(), ws) and torch.equal(raw(q).cpu(), raw(wq.contiguous()))
    assert torch.isfinite(s).all() and ((s > 0).all() if top >= 2.0 ** -117 else True)


def sorted_rows(T, E, K, seed, drop):
    g = torch.Generator().manual_seed(seed)
    idx = torch.randint(0, E, (T, K), generator=g, dtype=torch.int32)
    idx[torch.rand(T, K, generator=g) < drop] = -1
    return [torch.tensor(t, dtype=torch.int32) for t in ref.rows(idx, E)]


def want_cols(x, offsets, blocks, P):
    """Codes [c, 128 P] and scale [P, c] of the sorted rows x, and which blocks there are."""
    c = x.shape[1]
    q, s = torch.zeros(c, P * 128, dtype=torch.uint8), torch.zeros(P, c)
    for e in range(len(offsets) - 1):
        for b in range(int(blocks[e]), int(blocks[e + 1])):
            r = int(offsets[e]) + (b - int(blocks[e])) * 128
            part = x[r:min(r + 128, int(offsets[e + 1]))].float()
            cq, cs = ref.codes(part, (0,))
            q[:, b * 128:b * 128 + len(part)], s[b] = raw(cq.t().contiguous()), cs[0]
    return q, s, int(blocks[-1])


@pytest.mark.parametrize("T,c,E,K", [(1, 16, 1, 1), (1, 64, 8, 2), (50, 80, 8, 2), (128, 64, 1, 1), (129, 128, 1, 1), (300, 272, 4, 3),
                                     (1000, 1040, 64, 6), (4000, 96, 2, 2)])
@pytest.mark.parametrize("gather", [False, True])
def test_cols(T, c, E, K, gather):
    offsets, blocks, _, entry = sorted_rows(T, E, K, T + c, 0.2)
    R, P = T * K, eqb.eqb_expert_max_blocks(T * K, E) + 1
    x = values((T if gather else R, c), T).bfloat16()
    b, q = guarded8((c, P * 128))
    s = Guarded((P, c), torch.float32, fill=-3.0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    eqb.eqb_quant_cols(x.cuda(), offsets.cuda(), blocks.cuda(), entry=entry.cuda() if gather else None, K=K, q=q, scale=s.view, err_flag=err)
    torch.cuda.synchronize()
    assert b.intact() and s.intact() and err.item() == 0
    by_row = x[entry.long().clamp(min=0).div(K, rounding_mode="floor")] if gather else x
    wq, ws, n = want_cols(by_row, offsets, blocks, P)
    assert torch.equal(s.view.cpu()[:n], ws[:n]) and (s.view.cpu()[n:] == -3.0).all()
    got = raw(q).cpu()
    assert torch.equal(got[:, :n * 128], wq[:, :n * 128]) and (got[:, n * 128:] == 0x55).all()


def test_cols_with_tables_that_lie():
    """Whatever the device tables say, nothing outside the buffers is read or written."""
    x = values((100, 64), 1).bfloat16().cuda()
    for off, blk in (([0, 1000], [0, 8]), ([-500, 50], [0, 2]), ([90, 10], [0, 1]), ([0, 100], [0, 50])):
        b, q = guarded8((64, 2 * 128))
        s = Guarded((2, 64), torch.float32)
        eqb.eqb_quant_cols(x, torch.tensor(off, dtype=torch.int32, device="cuda"), torch.tensor(blk, dtype=torch.int32, device="cuda"),
                           q=q, scale=s.view)
        torch.cuda.synchronize()
        assert b.intact() and s.intact()
    entry = torch.tensor([5, 99, 100, -1, 2 ** 31 - 1, 199, 200, -2 ** 31], dtype=torch.int32, device="cuda")
    b, q = guarded8((64, 128))
    s = Guarded((1, 64), torch.float32)
    eqb.eqb_quant_cols(x, torch.tensor([0, 8], dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
                       entry=entry, K=2, q=q, scale=s.view)
    torch.cuda.synchronize()
    rows = torch.zeros(8, 64)
    for i, t in ((0, 2), (1, 49), (2, 50), (5, 99)):
        rows[i] = x[t].cpu().float()
    wq, ws = ref.codes(rows, (0,))
    assert torch.equal(s.view.cpu()[0], ws[0]) and torch.equal(raw(q).cpu()[:, :8], raw(wq.t().contiguous()))
    assert not raw(q).cpu()[:, 8:].any()


@pytest.mark.parametrize("E,n,d", [(1, 16, 16), (2, 128, 128), (3, 144, 272), (2, 1024, 48), (5, 336, 640), (1, 16, 4096)])
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("turned", [False, True])
def test_blocks(E, n, d, fp32, turned):
    w = values((E, n, d), n + d)
    w = w if fp32 else w.bfloat16()
    got = eqb.eqb_quant_blocks(w.cuda(), turned=turned)
    nb, db = (n + 127) // 128, (d + 127) // 128
    wq, ws = ref.codes(padded(w.float(), 1, 2).view(E, nb, 128, db, 128), (2, 4))
    wq, ws = wq.reshape(E, nb * 128, db * 128)[:, :n, :d].contiguous(), ws[:, :, 0, :, 0]
    assert torch.equal(got[1].cpu(), ws) and torch.equal(raw(got[0]).cpu(), raw(wq))
    assert near(got[0].cpu(), ref.spread(ref.spread(ws, 1, n), 2, d), w)
    if turned:
        assert torch.equal(got[3].cpu(), ws.transpose(1, 2)) and torch.equal(raw(got[2]).cpu(), raw(wq).transpose(1, 2))


def test_blocks_within_their_buffers():
    w = values((3, 144, 272), 1).cuda()
    (b0, q), (b1, qt) = guarded8((3, 144, 272)), guarded8((3, 272, 144))
    s, st = Guarded((3, 2, 3), torch.float32), Guarded((3, 3, 2), torch.float32)
    eqb.eqb_quant_blocks(w, q=q, scale=s.view, q_t=qt, scale_t=st.view)
    torch.cuda.synchronize()
    assert b0.intact() and b1.intact() and s.intact() and st.intact()


def test_nothing_to_do():
    q, s = eqb.eqb_quant_rows(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"))
    assert q.shape == (0, 64) and s.shape == (0, 1)
    off = torch.zeros(5, dtype=torch.int32, device="cuda")
    q, s = eqb.eqb_quant_cols(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), off, off)
    assert q.shape == (64, 0) and s.shape == (0, 64)
    q, s = eqb.eqb_quant_blocks(torch.empty(0, 64, 64, device="cuda"))
    assert q.shape == (0, 64, 64)


def test_refusals():
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(eqb.EqbError, match="UNSUPPORTED"):
        eqb.eqb_quant_rows(torch.zeros(4, 40, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError, match="bfloat16"):
        eqb.eqb_quant_rows(x.float())
    with pytest.raises(ValueError, match="shape"):
        eqb.eqb_quant_rows(x, q=torch.empty(5, 64, dtype=E4M3, device="cuda"))
    with pytest.raises(ValueError, match="contiguous"):
        eqb.eqb_quant_rows(x[:, :32])
    with pytest.raises(ValueError, match="shape"):
        eqb.eqb_quant_rows(x, slot=torch.zeros(5, 2, dtype=torch.int32, device="cuda"))
