"""EqbAdamW against the 64-bit plain form.

m and v are sums of two products in fp32: 4 roundings of 2^-24 of their terms.
The update divides two such values and adds eps: 16 roundings of its size; p has
two roundings of its own, and one to bf16 (2^-8 of itself).  In 8 bits a value is
off by half a step, 2^-4 of itself or 2^-10 scales, and the scale by 2^-22."""
import numpy as np
import pytest
import torch

import paper_2609_28053_gb300 as eqb
from gpu_harness import Guarded
from train_reference import adamw

pytestmark = pytest.mark.gpu

H = dict(lr=1e-2, step=3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
ULP = 2.0 ** -24


def ref(p, g, m, v, h=H):
    return adamw(p, g, m, v, h["lr"], h["step"], h["beta1"], h["beta2"], h["eps"], h["weight_decay"])


def check32(p0, g, m0, v0, p, m, v, h=H, bf16=False):
    rp, rm, rv = ref(p0, g, m0, v0, h)
    upd = np.abs(rp - p0 * (1 - h["lr"] * h["weight_decay"]))
    assert np.all(np.abs(m - rm) <= 4 * ULP * (np.abs(m0) + np.abs(g)) + 1e-44)
    assert np.all(np.abs(v - rv) <= 6 * ULP * (v0 + g.astype(np.float64) ** 2) + 1e-44)
    # m may cancel: its error is one of its terms
    terms = (np.abs(m0) + np.abs(g)) / np.maximum(np.abs(rm), 1e-300)
    tol = 3 * ULP * np.abs(p0) + upd * ULP * (16 + 4 * terms) + 1e-30
    assert np.all(np.abs(p - rp) <= tol + (2.0 ** -8 * np.abs(rp) * 1.01 if bf16 else 0))


def draw(n, seed):
    rng = np.random.default_rng(seed)
    p = (0.02 * rng.standard_normal(n)).astype(np.float32)
    g = (1e-3 * rng.standard_normal(n) * np.exp(rng.standard_normal(n))).astype(np.float32)
    m = (3e-4 * rng.standard_normal(n)).astype(np.float32)
    v = ((1e-3 * rng.standard_normal(n)) ** 2).astype(np.float32)
    return p, g, m, v


SIZES = [1, 3, 255, 256, 257, 0, 1024, 8191, 8192, 8193, 33000]


def guarded(a, dtype, shift):
    """A device copy of `a` with canaries around it, `shift` elements past a 16-byte boundary."""
    b = Guarded((len(a) + shift,), dtype, canary=-3.0)
    b.view[shift:].copy_(torch.from_numpy(a))
    if shift:
        b.view[:shift].fill_(-3.0)
    return b, b.view[shift:]


@pytest.mark.parametrize("pt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [0, 1])
def test_32_bits(pt, gt, shift):
    data = [draw(n, 10 + n) for n in SIZES]
    held = [[guarded(a, t, shift) for a, t in zip(d, (pt, gt, torch.float32, torch.float32))] for d in data]
    copies = [guarded(np.zeros(n, np.float32), torch.bfloat16, shift) for n in SIZES] if pt is torch.float32 else None
    before = [[v.float().cpu().numpy().copy() for _, v in h] for h in held]
    opt = eqb.EqbAdamW([h[0][1] for h in held], exp_avg=[h[2][1] for h in held], exp_avg_sq=[h[3][1] for h in held],
                       copies=copies and [c[1] for c in copies])
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    opt.step([h[1][1] for h in held], err_flag=err, **H)
    torch.cuda.synchronize()
    assert err.item() == 0
    for i, (h, b) in enumerate(zip(held, before)):
        assert all(x.intact() for x, _ in h)
        if shift:
            assert all(bool((x.view[:shift] == -3.0).all()) for x, _ in h)
        p, g, m, v = (x.float().cpu().numpy().astype(np.float64) for _, x in h)
        assert np.array_equal(g, b[1])
        check32(*[a.astype(np.float64) for a in (b[0], b[1], b[2], b[3])], p, m, v, bf16=pt is torch.bfloat16)
        if copies:
            assert copies[i][0].intact()
            assert torch.equal(copies[i][1], h[0][1].bfloat16())


def dec(codes, scale):
    """The values that 8-bit codes stand for."""
    s = scale.double().repeat_interleave(256)[:codes.numel()]
    return (codes.double() * s).cpu().numpy()


def check_codes(got, want, scale, root):
    """Half a step from the value, and the scale is the block's largest magnitude / 448."""
    n = len(want)
    s = scale.double().cpu().numpy()
    for b in range((n + 255) // 256):
        w, g = want[256 * b:256 * b + 256], got[256 * b:256 * b + 256]
        top = np.abs(w).max()
        assert abs(s[b] - top / 448) <= 2.0 ** -21 * top / 448
        tol = np.maximum(np.abs(w) * 2.0 ** -4, s[b] * 2.0 ** -10) * 1.001
        if root:
            low = (w > 0) & (w < s[b] * 2.0 ** -9)
            assert np.all(g[w > s[b] * 2.0 ** -20] > 0)
            tol = np.where(low, s[b] * 2.0 ** -9, tol)
        assert np.all(np.abs(g - w) <= tol + 1e-44)


@pytest.mark.parametrize("pt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [0, 1])
def test_8_bits(pt, gt, shift):
    """Three steps from zero states; before each the 64-bit form starts from what is stored."""
    data = [draw(n, 70 + n) for n in SIZES]
    ps = [guarded(d[0], pt, shift) for d in data]
    gs = [guarded(d[1], gt, shift) for d in data]
    ms = [Guarded((n + shift,), torch.uint8, canary=77) for n in SIZES]
    vs = [Guarded((n + shift,), torch.uint8, canary=77) for n in SIZES]
    f8 = torch.float8_e4m3fn
    opt = eqb.EqbAdamW([p[1] for p in ps], state_bits=8, exp_avg=[m.view[shift:].view(f8) for m in ms],
                       exp_avg_sq=[v.view[shift:].view(f8) for v in vs])
    for step in range(1, 4):
        h = dict(H, step=step)
        before = [(p[1].float().cpu().numpy().astype(np.float64), dec(opt.exp_avg[i].float(), opt.avg_scale[i]),
                   dec(opt.exp_avg_sq[i].float(), opt.sq_scale[i]) ** 2) for i, p in enumerate(ps)]
        opt.step([g[1] for g in gs], **h)
        torch.cuda.synchronize()
        for i, n in enumerate(SIZES):
            assert ps[i][0].intact() and ms[i].intact() and vs[i].intact()
            if n == 0:
                continue
            p0, m0, v0 = before[i]
            g = gs[i][1].float().cpu().numpy().astype(np.float64)
            rp, rm, rv = ref(p0, g, m0, v0, h)
            upd = np.abs(rp - p0 * (1 - h["lr"] * h["weight_decay"]))
            p = ps[i][1].float().cpu().numpy().astype(np.float64)
            terms = (np.abs(m0) + np.abs(g)) / np.maximum(np.abs(rm), 1e-300)
            tol = 3 * ULP * np.abs(p0) + upd * ULP * (24 + 4 * terms) + 1e-30
            assert np.all(np.abs(p - rp) <= tol + (2.0 ** -8 * np.abs(rp) * 1.01 if pt is torch.bfloat16 else 0))
            check_codes(dec(opt.exp_avg[i].float(), opt.avg_scale[i]), rm, opt.avg_scale[i], False)
            check_codes(dec(opt.exp_avg_sq[i].float(), opt.sq_scale[i]), np.sqrt(rv), opt.sq_scale[i], True)


def test_8_bits_wide_range_and_zero_blocks():
    """Roots over seven decades keep a positive code; blocks of zeros and of
    magnitudes below the normal numbers are stored as zeros."""
    n = 4 * 256
    g = np.zeros(n, np.float32)
    g[:256] = np.logspace(-7, 0, 256)
    g[512:768] = 1e-40
    g[768:] = 1e30
    p = torch.zeros(n, device="cuda")
    opt = eqb.EqbAdamW([p], state_bits=8)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    opt.step([torch.from_numpy(g).cuda()], err_flag=err, **dict(H, step=1, weight_decay=0.0))
    torch.cuda.synchronize()
    q = opt.exp_avg_sq[0].float().cpu().numpy()
    assert np.all(q[:256] > 0) and not q[256:768].any()
    assert opt.sq_scale[0][1] == 0 and opt.avg_scale[0][1] == 0 and opt.sq_scale[0][2] == 0
    # a first step moves by lr whatever the gradient's size (eps aside)
    assert np.allclose(p[128:256].cpu().numpy(), -H["lr"], rtol=1e-3)
    assert not p[256:512].any()
    assert err.item() == 4  # 1e60 is beyond fp32: the last block's second moment


@pytest.mark.parametrize("bits", [8, 32])
def test_grad_scale_none_and_many_tensors(bits):
    """More tensors than a launch takes, some without a gradient; the scale acts as if the gradient had been multiplied."""
    rng = np.random.default_rng(3)
    count = 900
    sizes = rng.integers(0, 700, count)
    p0 = [torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda() for n in sizes]
    g0 = [torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda() for n in sizes]
    a, b = [t.clone() for t in p0], [t.clone() for t in p0]
    oa, ob = eqb.EqbAdamW(a, state_bits=bits), eqb.EqbAdamW(b, state_bits=bits)
    skip = set(range(0, count, 11))
    oa.step([None if i in skip else g for i, g in enumerate(g0)], grad_scale=torch.tensor([0.25], device="cuda"), **H)
    ob.step([torch.zeros_like(g) if i in skip else g * 0.25 for i, g in enumerate(g0)], **H)
    torch.cuda.synchronize()
    for i in range(count):
        assert torch.equal(a[i], p0[i] if i in skip else b[i])
        if i not in skip:
            assert torch.equal(oa.exp_avg[i].float(), ob.exp_avg[i].float())
            assert torch.equal(oa.exp_avg_sq[i].float(), ob.exp_avg_sq[i].float())
        else:
            assert not oa.exp_avg[i].float().any()


def test_shapes_streams_and_repeated_steps():
    """Matrices, another stream, ten steps against the 64-bit form carried along."""
    rng = np.random.default_rng(5)
    p0 = rng.standard_normal((37, 64)).astype(np.float32)
    p = torch.from_numpy(p0.copy()).cuda()
    c = torch.empty(37, 64, dtype=torch.bfloat16, device="cuda")
    opt = eqb.EqbAdamW([p], copies=[c])
    rp, rm, rv = p0.astype(np.float64), np.zeros((37, 64)), np.zeros((37, 64))
    gs = [rng.standard_normal((37, 64)).astype(np.float32) for _ in range(10)]
    dev = [torch.from_numpy(g).cuda() for g in gs]
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    for k in range(10):
        opt.step([dev[k]], stream=st, **dict(H, step=k + 1))
        rp, rm, rv = ref(rp, gs[k], rm, rv, dict(H, step=k + 1))
    st.synchronize()
    assert np.allclose(p.cpu().numpy(), rp, rtol=2e-5, atol=2e-6)
    assert torch.equal(c, p.bfloat16())


@pytest.mark.parametrize("bits", [8, 32])
def test_non_finite_gradient_is_flagged(bits):
    for bad in (float("nan"), float("inf")):
        p = torch.ones(1000, device="cuda")
        g = torch.ones(1000, device="cuda")
        g[513] = bad
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        opt = eqb.EqbAdamW([p], state_bits=bits)
        opt.step([g], err_flag=err, **H)
        assert err.item() == 4


def test_refusals():
    p = torch.zeros(8, device="cuda")
    g = torch.zeros(8, device="cuda")
    opt = eqb.EqbAdamW([p])
    with pytest.raises(ValueError, match="entries"):
        opt.step([], lr=1e-3, step=1)
    with pytest.raises(TypeError, match="grads"):
        opt.step([g.double()], lr=1e-3, step=1)
    with pytest.raises(ValueError, match="shape"):
        opt.step([g[:4]], lr=1e-3, step=1)
    with pytest.raises(ValueError, match="contiguous"):
        opt.step([torch.zeros(16, device="cuda")[::2]], lr=1e-3, step=1)
    for kw in (dict(lr=-1.0, step=1), dict(lr=1e-3, step=0), dict(lr=1e-3, step=1, beta1=1.0), dict(lr=1e-3, step=1, eps=0.0)):
        with pytest.raises(eqb.EqbError):
            opt.step([g], **kw)
    p.data = torch.zeros(8, device="cuda")
    with pytest.raises(ValueError, match="moved"):
        opt.step([g], lr=1e-3, step=1)
    with pytest.raises(TypeError, match="copies"):
        eqb.EqbAdamW([p.bfloat16()], copies=[p.bfloat16()])
    with pytest.raises(ValueError, match="state_bits"):
        eqb.EqbAdamW([p], state_bits=16)
