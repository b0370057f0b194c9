"""eqb_router_grad's forms of launch: both gradients in two launches and in one,
either alone, written and added to, from one thread and from two.  Whole numbers,
so every form has the same, exact sums."""
import threading

import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu

ONE_LAUNCH = 1 << 27  # elements of x up to which both gradients, written, share a launch


def whole(n, m, top, g):
    return torch.randint(-top, top + 1, (n, m), generator=g, device="cuda", dtype=torch.int16).bfloat16()


def case(T, d, E, add=False, want=("dx", "dW"), seed=0):
    """Outputs, what they have to be, and a call that forms them anew."""
    g = torch.Generator(device="cuda").manual_seed(seed + T + d + E)
    dz, x, W = whole(T, E, 1, g), whole(T, d, 2, g), whole(E, d, 2, g)
    dx0, dW0 = whole(T, d, 50, g), whole(E, d, 50, g).float()
    dx = torch.zeros_like(dx0) if "dx" in want else None
    dW = torch.zeros_like(dW0) if "dW" in want else None
    ws = torch.empty(max(1, eqb.eqb_router_grad_workspace_bytes(T, d, E)), dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    right = []
    if dx is not None:
        right.append((dx, (dz.float() @ W.float() + (dx0.float() if add else 0.0)).bfloat16()))
    if dW is not None:
        right.append((dW, (dz.double().t() @ x.double() + (dW0.double() if add else 0.0)).float()))

    def call():
        if add:
            for t, t0 in ((dx, dx0), (dW, dW0)):
                if t is not None:
                    t.copy_(t0)
        eqb.eqb_router_grad(dz, x, W, dx=dx, dW=dW, accumulate_dx=add, accumulate_dW=add, workspace=ws, err_flag=err)

    def check():
        assert err.item() == 0
        for got, w in right:
            assert torch.equal(got, w)
    return call, check


@pytest.mark.parametrize("T,d,E", [(2049, 512, 144), (3001, 704, 256), (5000, 64, 256), (70000, 1024, 256), (20000, 2048, 128)])
@pytest.mark.parametrize("want", [("dW",), ("dx",), ("dx", "dW")])
@pytest.mark.parametrize("add", [False, True])
def test_each_output_alone_and_both(T, d, E, want, add):
    """dW in parts, of one and of two groups of experts."""
    call, check = case(T, d, E, add, want)
    call()
    check()


@pytest.mark.parametrize("E", [64, 128, 256])
def test_two_launches(E):
    T, d = 40000, 4096
    assert T * d > ONE_LAUNCH
    call, check = case(T, d, E)
    call()
    check()


@pytest.mark.parametrize("T,d,E,add", [(40000, 4096, 128, False), (20000, 2048, 128, True), (900, 1024, 256, True)])
def test_first_call_of_a_thread(T, d, E, add):
    call, check = case(T, d, E, add)
    failed = []

    def work():
        try:
            call()
        except Exception as e:
            failed.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    check()


@pytest.mark.parametrize("small,large", [
    ((40000, 4096, 64, False), (40000, 4096, 256, False)),  # two launches each
    ((300, 256, 64, True), (900, 1024, 256, True)),         # one launch each, added to
    ((20000, 2048, 64, True), (30000, 2048, 256, True)),    # the same, dW in parts
    ((40000, 4096, 128, False), (20000, 2048, 128, True))])
def test_two_shapes_from_two_threads(small, large):
    cases = [case(*small), case(*large, seed=1)]
    torch.cuda.synchronize()
    failed = []

    def work(call):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(60):
                    call()
                torch.cuda.current_stream().synchronize()
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=(call,)) for call, _ in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for _, check in cases:
        check()
