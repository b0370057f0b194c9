"""The training operators from host threads: a thread's first CUDA work, and two
shapes at once on two streams."""
import threading

import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


def grad(T, d, E, add=False):
    dz = torch.randint(-2, 3, (T, E), device="cuda").bfloat16()
    x = torch.randint(-2, 3, (T, d), device="cuda").bfloat16()
    W = torch.randint(-2, 3, (E, d), device="cuda").bfloat16()
    out = [torch.zeros(T, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(E, d, device="cuda")]
    ws = torch.empty(eqb.eqb_router_grad_workspace_bytes(T, d, E), dtype=torch.uint8, device="cuda")
    return out, lambda: eqb.eqb_router_grad(dz, x, W, dx=out[0], dW=out[1], workspace=ws)


def loss(T, E, M):
    z = torch.randn(T, E, device="cuda").bfloat16()
    idx = torch.randint(0, E, (T, 4), dtype=torch.int32, device="cuda")
    off = torch.arange(M + 1, device="cuda") * T // M
    out = [torch.zeros(M, 2, device="cuda"), torch.zeros(T, E, device="cuda"), torch.zeros(M, E, dtype=torch.int32, device="cuda")]
    ws = torch.empty(eqb.eqb_balance_loss_workspace_bytes(T, E, M), dtype=torch.uint8, device="cuda")
    return out, lambda: eqb.eqb_balance_loss(z, idx, off, 0.1, grad_out=out[1], counts=out[2], loss=out[0], workspace=ws)


def adam(count, n, bits):
    out = [torch.randn(n, device="cuda") for _ in range(count)]
    g = [torch.randn(n, device="cuda") for _ in range(count)]
    opt = eqb.EqbAdamW(out, state_bits=bits)
    p0 = [t.clone() for t in out]
    states = opt.exp_avg + opt.exp_avg_sq + (opt.avg_scale or []) + (opt.sq_scale or [])

    def f():  # a first step each time
        for t, p in zip(out, p0):
            t.copy_(p)
        for t in states:
            t.zero_()
        opt.step(g, lr=1e-3, step=1)
    return out, f


@pytest.mark.parametrize("make,args", [(grad, (300, 256, 64)), (grad, (20000, 4096, 128)), (loss, (500, 64, 2)), (loss, (60000, 256, 3)),
                                       (adam, (3, 1000, 8))])
def test_first_call_of_a_thread(make, args):
    out, f = make(*args)
    f()
    torch.cuda.synchronize()
    ref, failed = [t.clone() for t in out], []
    for t in out:
        t.zero_()

    def work():
        try:
            f()
        except Exception as e:
            failed.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    assert all(torch.equal(x, y) for x, y in zip(out, ref))


@pytest.mark.parametrize("make,small,large", [
    (grad, (300, 256, 64), (900, 1024, 256)),       # one launch, two rings
    (grad, (20000, 4096, 64), (20000, 4096, 256)),  # two launches
    (loss, (500, 64, 2), (4000, 64, 2)),            # clusters
    (loss, (30000, 256, 2), (60000, 200, 900)),     # blocks of eight warps, and of fewer
    (adam, (3, 1000, 8), (20, 30000, 8))])
def test_two_shapes_from_two_threads(make, small, large):
    calls = [make(*small), make(*large)]
    refs = []
    for out, f in calls:
        f()
        torch.cuda.synchronize()
        refs.append([t.clone() for t in out])
    failed = []

    def work(f):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(200):
                    f()
                torch.cuda.current_stream().synchronize()
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=(f,)) for _, f in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for (out, _), ref in zip(calls, refs):
        assert all(torch.equal(x, y) for x, y in zip(out, ref))
