"""eqb_balance_loss against the 64-bit plain form.

Tolerances.  A probability is off by the exponential's 2 ulps, its argument's
rounding (|z - max| log2(e) 2^-24, logits within 20 of the maximum: 1.2e-6), the
reciprocal and the sums over at most 1,024 experts: below 5e-6 of itself in all.
The gradient is p times a difference whose terms are as far off: 2e-5 of the
magnitude of its terms, plus the output's rounding.  Loss and mean probability
are sums of non-negative terms: 1e-5 of themselves."""
import numpy as np
import pytest
import torch

import paper_2609_28053_gb300 as eqb
from gpu_harness import Guarded
from train_reference import balance

pytestmark = pytest.mark.gpu


def make(T, E, K, M, seed, ragged=False, masked=False, holes=False, dtype=torch.bfloat16, low=0.0):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((rng.standard_normal((T, E)) * 2 + low).astype(np.float32)).to(dtype)
    idx = np.argsort(rng.random((T, E)), axis=1)[:, :K].astype(np.int32)
    if ragged:
        off = np.concatenate([[0], np.sort(rng.integers(0, T + 1, M - 1)), [T]]).astype(np.int64)
    else:
        off = np.array([T * l // M for l in range(M + 1)], np.int64)
    mask = rng.random(T) < 0.7 if masked else None
    if masked:
        z[torch.from_numpy(~mask)] = float("nan")
    if holes:
        z[::3, 1] = -float("inf")
        z[5::17] = -float("inf")
        if masked:
            mask[5::17] = True
        idx[::4, 0] = -1
        idx[1::9, K - 1] = E + 3
    return z, idx, off, mask, rng


def run(z, idx, off, mask, score, alpha, zeta, grad="fp32", add=False, scale=None, rng=None, want_prob=True):
    T, E = z.shape
    M = len(off) - 1
    K = idx.shape[1]
    dev = "cuda"
    gi = torch.from_numpy((1e-4 * rng.standard_normal((T, E))).astype(np.float32)).to(dev) if add else None
    go = {"none": None, "fp32": Guarded((T, E), torch.float32, fill=7.0),
          "bf16": Guarded((T, E), torch.bfloat16, fill=7.0, canary=-3.0)}[grad]
    counts, loss, prob = Guarded((M, E), torch.int32, fill=99), Guarded((M, 2), torch.float32, fill=9.0), \
        Guarded((M, E), torch.float32, fill=9.0)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    ws = torch.full((eqb.eqb_balance_loss_workspace_bytes(T, E, M),), 0xff, dtype=torch.uint8, device=dev)
    eqb.eqb_balance_loss(z.to(dev), torch.from_numpy(idx).to(dev), torch.from_numpy(off).to(dev), alpha, zeta=zeta,
                         score=score, mask=None if mask is None else torch.from_numpy(mask).to(dev), grad_in=gi,
                         grad_out=None if go is None else go.view,
                         grad_scale=None if scale is None else torch.tensor([scale], device=dev),
                         counts=counts.view, prob=prob.view if want_prob else None, loss=loss.view, workspace=ws, err_flag=err)
    torch.cuda.synchronize()
    for b in (counts, loss, prob, go):
        assert b is None or b.intact()
    return counts.view.cpu().numpy(), loss.view.cpu().numpy(), prob.view.cpu().numpy(), \
        None if go is None else go.view.float().cpu().numpy(), None if gi is None else gi.cpu().numpy(), err.item()


def check(z, idx, off, mask, score, alpha, zeta, out, scale=1.0, bf16=False, want_prob=True):
    counts, loss, prob, grad, gi, err = out
    zz = z.double().numpy()
    r_loss, r_counts, r_prob, r_grad, size = balance(zz, idx, off, score, alpha, zeta, mask)
    assert err == 0
    assert np.array_equal(counts, r_counts)
    assert np.all(np.abs(loss - r_loss) <= 1e-5 * np.abs(r_loss) + 1e-30)
    if want_prob:
        assert np.all(np.abs(prob - r_prob) <= 1e-5 * r_prob + 1e-30)
    if grad is None:
        return
    want = r_grad * scale + (0.0 if gi is None else gi.astype(np.float64))
    tol = 2e-5 * size * abs(scale) + 2.0 ** -22 * np.abs(want) + 1e-30
    if gi is not None:
        tol += 2.0 ** -23 * np.abs(gi)
    if bf16:
        tol = tol * 1.01 + 2.0 ** -8 * np.abs(want)
    bad = np.abs(grad - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:3], grad[bad][:3], want[bad][:3])


@pytest.mark.parametrize("E,K", [(8, 2), (16, 1), (40, 6), (64, 8), (96, 6), (128, 8), (256, 8), (264, 6), (384, 8),
                                 (520, 4), (768, 8), (1024, 31)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_widths(E, K, score):
    z, idx, off, mask, rng = make(173, E, K, 3, 100 + E)
    zeta = 1e-3 if score == "softmax" else 0.0
    check(z, idx, off, mask, score, 0.1, zeta, run(z, idx, off, mask, score, 0.1, zeta, rng=rng))


@pytest.mark.parametrize("T", [1, 2, 31, 64, 65, 1000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("grad,add", [("none", False), ("fp32", False), ("fp32", True), ("bf16", False), ("bf16", True)])
def test_lengths_types_and_outputs(T, dtype, grad, add):
    z, idx, off, mask, rng = make(T, 64, 4, min(T, 5), T, ragged=True, dtype=dtype)
    for score, zeta in (("softmax", 0.01), ("softmax", 0.0), ("sigmoid", 0.0)):
        out = run(z, idx, off, mask, score, 0.3, zeta, grad, add, 64.0 if grad != "none" else None, rng)
        check(z, idx, off, mask, score, 0.3, zeta, out, 64.0, grad == "bf16")


@pytest.mark.parametrize("E", [8, 96, 256, 512])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masks_closed_experts_and_empty_rows(E, score, dtype):
    """NaN in masked rows, -inf logits, rows of -inf, lists with -1 and numbers
    past E, empty microbatches, microbatches without a valid token."""
    z, idx, off, mask, rng = make(400, E, 4, 60, E, ragged=True, masked=True, holes=True, dtype=dtype)
    mask[off[3]:off[9]] = False
    zeta = 1e-3 if score == "softmax" else 0.0
    out = run(z, idx, off, mask, score, 0.1, zeta, "fp32", True, rng=rng)
    check(z, idx, off, mask, score, 0.1, zeta, out)
    assert np.array_equal(out[3][~mask], out[4][~mask])  # a masked token's gradient is what it was
    out = run(z, idx, off, mask, score, 0.1, zeta, "bf16", False, rng=rng)
    check(z, idx, off, mask, score, 0.1, zeta, out, 1.0, True)
    assert not out[3][~mask].any()


@pytest.mark.parametrize("low", [-60.0, -200.0, 30.0])
def test_sigmoid_far_from_zero(low):
    """All sigmoids tiny (their ratios count) or all near one."""
    z, idx, off, mask, rng = make(90, 128, 8, 2, 5, low=low, dtype=torch.float32)
    if low > 0:
        z = z.clamp(max=32.0)
    # (1 - s) near one is formed as a product, so it keeps its relative accuracy; the
    # argument of the exponential is as large as |z| here: 200 log2(e) 2^-24 ln 2 = 1.2e-5
    counts, loss, prob, grad, _, err = run(z, idx, off, mask, "sigmoid", 0.1, 0.0, rng=rng)
    r_loss, r_counts, r_prob, r_grad, size = balance(z.double().numpy(), idx, off, "sigmoid", 0.1, 0.0)
    s = 1.0 / (1.0 + np.exp(-z.double().numpy()))
    size = np.where(s > 0.5, size / np.maximum(1 - s, 1e-300) * np.exp(-z.double().numpy()), size)
    assert err == 0 and np.array_equal(counts, r_counts)
    assert np.all(np.abs(loss - r_loss) <= 4e-5 * np.abs(r_loss))
    assert np.all(np.abs(prob - r_prob) <= 4e-5 * r_prob)
    if low < 0:
        assert np.all(np.abs(grad - r_grad) <= 8e-5 * size + 1e-30)
    else:  # 1 - s from 64-bit sigmoids would cancel: take it as exp(-z) s
        zz = z.double().numpy()
        F = r_counts / (8 * np.diff(off)[:, None])
        Ft = np.repeat(F, np.diff(off), axis=0)
        p = s / s.sum(1, keepdims=True)
        want = 0.1 / np.repeat(np.diff(off), np.diff(off))[:, None] * p * (Ft - (p * Ft).sum(1, keepdims=True)) * np.exp(-zz) * s
        assert np.all(np.abs(grad - want) <= 8e-5 * size + 1e-30)


def test_gradient_against_differences():
    """The 64-bit loss with its counts held, differenced at h = 1e-4: the error
    h^2 / 6 times a third derivative of at most the loss's own size."""
    z, idx, off, mask, rng = make(12, 16, 3, 2, 9, dtype=torch.float32)
    for score, zeta in (("softmax", 0.02), ("sigmoid", 0.0)):
        grad = run(z, idx, off, mask, score, 0.5, zeta, rng=rng)[3]
        zz = z.double().numpy()
        f = balance(zz, idx, off, score, 0.5, zeta)[1]
        h = 1e-4
        for t, e in [(0, 0), (3, 7), (6, 15), (11, 2)]:
            a, b = zz.copy(), zz.copy()
            a[t, e] += h
            b[t, e] -= h
            d = (balance(a, idx, off, score, 0.5, zeta, counts=f)[0].sum() -
                 balance(b, idx, off, score, 0.5, zeta, counts=f)[0].sum()) / (2 * h)
            assert abs(d - grad[t, e]) <= 1e-7


def test_balanced_counts_give_a_zero_gradient():
    T, E, K = 64, 16, 4
    idx = ((np.arange(T)[:, None] * K + np.arange(K)) % E).astype(np.int32)
    z = torch.randn(T, E).bfloat16()
    off = np.array([0, T], np.int64)
    out = run(z, idx, off, None, "softmax", 0.1, 0.0, rng=np.random.default_rng(0))
    assert not out[3].any()
    assert abs(out[1][0, 0] - 0.1 / E) <= 1e-7


def test_same_bits_and_fewer_outputs():
    z, idx, off, mask, rng = make(5000, 256, 8, 7, 3, ragged=True)
    a = run(z, idx, off, mask, "softmax", 0.1, 1e-3, "fp32", rng=rng)
    b = run(z, idx, off, mask, "softmax", 0.1, 1e-3, "fp32", rng=rng)
    for x, y in zip(a[:4], b[:4]):
        assert np.array_equal(x, y)
    c = run(z, idx, off, mask, "softmax", 0.1, 1e-3, "none", rng=rng)
    assert np.array_equal(a[1], c[1]) and np.array_equal(a[2], c[2])
    d = run(z, idx, off, mask, "softmax", 0.1, 1e-3, "fp32", rng=rng, want_prob=False)
    assert np.array_equal(a[1], d[1]) and np.array_equal(a[3], d[3])


def test_in_place_and_another_stream():
    z, idx, off, mask, rng = make(300, 128, 8, 3, 4)
    dev = "cuda"
    g = torch.randn(300, 128, device=dev) * 1e-4
    want = torch.empty_like(g)
    args = (z.to(dev), torch.from_numpy(idx).to(dev), torch.from_numpy(off).to(dev), 0.1)
    eqb.eqb_balance_loss(*args, grad_in=g, grad_out=want)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    ws = torch.empty(eqb.eqb_balance_loss_workspace_bytes(300, 128, 3), dtype=torch.uint8, device=dev)
    loss, counts = eqb.eqb_balance_loss(*args, grad_in=g, grad_out=g, workspace=ws, stream=st)
    st.synchronize()
    assert torch.equal(g, want)


def test_no_tokens():
    for M in (1, 3):
        loss, counts = eqb.eqb_balance_loss(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"),
                                            torch.empty(0, 4, dtype=torch.int32, device="cuda"),
                                            torch.zeros(M + 1, dtype=torch.int64, device="cuda"), 0.1)
        torch.cuda.synchronize()
        assert not loss.any() and not counts.any()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_nan_is_flagged(score):
    z, idx, off, mask, rng = make(50, 64, 4, 2, 8)
    z[31, 5] = float("nan")
    assert run(z, idx, off, mask, score, 0.1, 0.0, rng=rng)[5] == 4
    if score == "softmax":
        z[31, 5] = float("inf")
        assert run(z, idx, off, mask, score, 0.1, 0.0, rng=rng)[5] == 4


def test_long_batch_counts():
    """Counts of a batch that many blocks share, against torch's."""
    T, E, K, M = 300001, 128, 8, 5
    idx = torch.randint(-1, E, (T, K), dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 5, 5, 100000, 250000, T], device="cuda")
    z = torch.randn(T, E, device="cuda").bfloat16()
    prob = torch.empty(M, E, device="cuda")
    loss, counts = eqb.eqb_balance_loss(z, idx, off, 0.1, prob=prob)
    p = torch.softmax(z.double(), 1)
    for l in range(M):
        ids = idx[off[l]:off[l + 1]].long().flatten()
        want = torch.bincount(ids[ids >= 0], minlength=E)
        assert torch.equal(counts[l].long(), want)
        if off[l + 1] > off[l]:
            P = p[off[l]:off[l + 1]].mean(0)
            assert torch.all((prob[l] - P).abs() <= 1e-5 * P)


@pytest.mark.parametrize("T,E,M,score,masked,grad", [(20000, 96, 70, "sigmoid", True, True), (20000, 256, 1900, "softmax", True, True),
                                                     (40000, 128, 5, "softmax", False, True), (300000, 128, 3, "sigmoid", True, False)])
def test_calls_one_after_the_other_in_the_same_buffers(T, E, M, score, masked, grad):
    """Calls of different inputs share counts and workspace with nothing between
    them: each gives the same bits as alone."""
    dev, sets = "cuda", []
    for seed in (1, 2, 3):
        z, idx, off, mask, rng = make(T, E, 6, M, seed, ragged=True)
        mask = torch.from_numpy(rng.random(T) < 0.2 * seed + 0.2).to(dev) if masked else None
        sets.append(dict(z=z.to(dev), idx=torch.from_numpy(idx).to(dev), off=torch.from_numpy(off).to(dev), mask=mask,
                         grad=torch.empty(T, E, device=dev) if grad else None, prob=torch.empty(M, E, device=dev),
                         loss=torch.empty(M, 2, device=dev)))
    counts = torch.empty(M, E, dtype=torch.int32, device=dev)
    ws = torch.empty(eqb.eqb_balance_loss_workspace_bytes(T, E, M), dtype=torch.uint8, device=dev)

    def call(s):
        eqb.eqb_balance_loss(s["z"], s["idx"], s["off"], 0.1, score=score, mask=s["mask"], grad_out=s["grad"], counts=counts,
                             prob=s["prob"], loss=s["loss"], workspace=ws)

    alone = []
    for s in sets:
        call(s)
        torch.cuda.synchronize()
        alone.append([None if s[k] is None else s[k].clone() for k in ("grad", "prob", "loss")])
    for _ in range(20):
        for s in sets:
            call(s)
    torch.cuda.synchronize()
    for s, want in zip(sets, alone):
        for k, w in zip(("grad", "prob", "loss"), want):
            assert w is None or torch.equal(s[k], w)
