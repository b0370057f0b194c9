"""Memory that a call allocates itself belongs to the stream that it launches on."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu

T, E, K, M, D = 3000, 64, 4, 3, 256


class Recorder:
    """The library, with the arguments of its calls kept."""

    def __init__(self, lib):
        self.lib, self.args = lib, []

    def __getattr__(self, name):
        fn = getattr(self.lib, name)

        def call(*args):
            self.args += args
            return fn(*args)
        return call


def made_on(ptr):
    """The stream whose memory an address lies in; None if it is not the allocator's."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= ptr < seg["address"] + seg["total_size"]:
            return seg["stream"]
    return None


def inputs():
    g = torch.Generator(device="cuda").manual_seed(7)
    z = torch.randn(T, E, generator=g, device="cuda").bfloat16()
    idx = torch.topk(z, K).indices.int()
    off = torch.arange(M + 1, device="cuda") * T // M
    x = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    W = torch.randn(E, D, generator=g, device="cuda").bfloat16()
    return z, idx, off, x, W


def calls(z, idx, off, x, W):
    b, b_next = torch.zeros(E, device="cuda"), torch.zeros(E, device="cuda")
    tau = eqb.eqb_route_topk(z, b, K)[1]
    loads = torch.zeros(M, E, dtype=torch.int32, device="cuda")
    loads += T * K // (M * E)
    dW = torch.empty(E, D, device="cuda")
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    ws = torch.zeros(max(eqb.eqb_layer_workspace_bytes(E), eqb.eqb_rank_averaged_workspace_bytes(E, 2)), dtype=torch.uint8,
                     device="cuda")
    return {
        "eqb_balance_loss": lambda s: eqb.eqb_balance_loss(z, idx, off, 0.1, mask=mask, stream=s),
        "eqb_router_grad": lambda s: eqb.eqb_router_grad(z, x, W, dW=dW, stream=s),
        "eqb_route_topk": lambda s: eqb.eqb_route_topk(z, b, K, stream=s),
        "eqb_router_logits": lambda s: eqb.eqb_router_logits(x, W, stream=s),
        "eqb_router_route": lambda s: eqb.eqb_router_route(x, W, b, K, stream=s),
        "lei_coefficients": lambda s: eqb.lei_coefficients(loads, off, K, 1e-3, 1.0, stream=s),
        "eqb_maxvio": lambda s: eqb.eqb_maxvio(loads, off, K, stream=s),
        "eqb_rank_averaged_bias": lambda s: eqb.eqb_rank_averaged_bias(z, tau, K, [0, 1000, T], ws, stream=s),
        "eqb_fixed_hist_bias": lambda s: eqb.eqb_fixed_hist_bias(z, tau, K, -4.0, 1 / 32, ws, stream=s),
        "eqb_layer_step": lambda s: eqb.eqb_layer_step(z, b, K, off, loads, b_next, ws, stream=s),
    }


NAMES = ["eqb_balance_loss", "eqb_router_grad", "eqb_route_topk", "eqb_router_logits", "eqb_router_route", "lei_coefficients",
         "eqb_maxvio", "eqb_rank_averaged_bias", "eqb_fixed_hist_bias", "eqb_layer_step"]


@pytest.mark.parametrize("name", NAMES)
def test_made_on_the_stream_of_the_call(name, monkeypatch):
    data = inputs()
    call = calls(*data)[name]
    st = torch.cuda.Stream()
    held = {b["address"] for seg in torch.cuda.memory_snapshot() for b in seg["blocks"] if b["state"] == "active_allocated"}
    lib = Recorder(eqb.load())
    monkeypatch.setattr(eqb, "load", lambda: lib)
    torch.cuda.synchronize()
    out = call(st)
    st.synchronize()
    made = {a for a in lib.args if type(a) is int and made_on(a) is not None} - held
    assert made, "the call allocates something"
    assert all(made_on(a) == st.cuda_stream for a in made)
    del out


@pytest.mark.parametrize("name", ["eqb_balance_loss", "eqb_router_grad"])
def test_workspaces_of_queued_calls_are_their_own(name):
    """Calls wait in a stream while another one takes memory of the workspaces' sizes and fills it."""
    data = inputs()
    call = calls(*data)[name]
    kept = []

    def run(s):
        out = call(s)
        kept.append([t.clone() for t in out if t is not None] if s is None else out)
    run(None)
    torch.cuda.synchronize()
    want = kept.pop()
    sizes = [eqb.eqb_balance_loss_workspace_bytes(T, E, M), eqb.eqb_router_grad_workspace_bytes(T, D, E)]
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        torch.cuda._sleep(2_000_000)
    for _ in range(60):
        run(st)
        for n in sizes:
            for _ in range(5):
                torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0xff)
    torch.cuda.synchronize()
    for out in kept:
        for a, b in zip([t for t in out if t is not None], want):
            assert torch.equal(a, b)
