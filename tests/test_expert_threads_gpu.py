"""The experts' calls from several threads, first calls of a thread among them, and on
streams that are not the current one."""
import threading

import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def product(R, n, d, E, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(-3, 4, (R, d), generator=g, device="cuda").float().to(E4M3)
    w = torch.randint(-2, 3, (E, n, d), generator=g, device="cuda").float().to(E4M3)
    s, ws = torch.ones(R, (d + 127) // 128, device="cuda"), torch.ones(E, (n + 127) // 128, (d + 127) // 128, device="cuda")
    off = torch.linspace(0, R, E + 1, device="cuda").int()
    want = torch.cat([q[a:b].float() @ w[e].float().t() for e, (a, b) in enumerate(zip(off.tolist(), off.tolist()[1:]))]).bfloat16()
    out = torch.empty_like(want)
    return (lambda: eqb.eqb_expert_matmul(q, s, w, ws, off, out=out)), (lambda: torch.equal(out, want))


def lists(T, E, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(T, E, generator=g, device="cuda")
    idx, w = torch.empty(T, K, dtype=torch.int32, device="cuda"), torch.empty(T, K, device="cuda")
    want = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :K].int()
    ws = torch.empty(max(eqb.eqb_expert_rows_workspace_bytes(T, K, E), 1), dtype=torch.uint8, device="cuda")
    order = torch.sort(want.flatten(), stable=True).indices
    got = [None]

    def call():
        eqb.eqb_gate_topk(z, None, K, topk_idx=idx, weight=w)
        got[0] = eqb.eqb_expert_rows(idx, E, workspace=ws)

    return call, (lambda: torch.equal(idx, want) and torch.equal(got[0][3].long(), order))


@pytest.mark.parametrize("cases", [
    (lambda: product(3000, 512, 256, 4, 1), lambda: product(20, 256, 512, 8, 2)),      # wide and narrow tiles
    (lambda: lists(20000, 256, 8, 3), lambda: lists(9000, 1000, 8, 4)),                # shared memory of different sizes
    (lambda: product(600, 640, 128, 40, 5), lambda: lists(70000, 64, 4, 6))])
def test_two_threads(cases):
    made = [c() for c in cases]
    torch.cuda.synchronize()
    failed = []

    def work(call):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(50):
                    call()
                torch.cuda.current_stream().synchronize()
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=(call,)) for call, _ in made]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    assert all(ok() for _, ok in made)


def test_a_stream_that_is_not_the_current_one():
    """The call's kernels and the memory that it makes itself are the given stream's."""
    s = torch.cuda.Stream()
    x = torch.randn(2000, 256, device="cuda").bfloat16()
    z = torch.randn(2000, 64, device="cuda")
    W = torch.randn(64, 128, 256, device="cuda")
    b = torch.zeros(64, device="cuda")

    def chain(stream):
        idx, w = eqb.eqb_gate_topk(z, b, 4, stream=stream)
        off, blk, slot, entry = eqb.eqb_expert_rows(idx, 64, stream=stream)
        q, sc = eqb.eqb_quant_rows(x, slot, stream=stream)
        wq, ws = eqb.eqb_quant_blocks(W, stream=stream)
        rows = eqb.eqb_expert_matmul(q, sc, wq, ws, off, stream=stream)
        y = eqb.eqb_expert_combine(rows, slot, w, stream=stream)
        g = torch.zeros_like(rows)
        s.wait_stream(torch.cuda.current_stream())
        g, gw = eqb.eqb_expert_combine_grad(y, rows, slot, w, grad_rows=g, grad_weight=torch.empty_like(w), stream=stream)
        a = eqb.eqb_quant_cols(g, off, blk, stream=stream)
        c = eqb.eqb_quant_cols(x, off, blk, entry, 4, stream=stream)
        return y, eqb.eqb_expert_wgrad(*a, *c, blk, stream=stream), eqb.eqb_gate_grad(z, idx, gw, stream=stream)

    want = chain(None)
    torch.cuda.synchronize()
    got = chain(s)
    s.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)
