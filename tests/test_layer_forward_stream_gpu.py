"""eqb_layer_forward on a stream that is not the current one: the workspace is
cleared there too, in order with the calls that use it."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


def test_calls_one_after_the_other_in_one_workspace():
    T, E, K, M = 200_000, 64, 6, 4
    g = torch.Generator(device="cuda").manual_seed(2)
    zs = [torch.randn(T, E, generator=g, device="cuda").bfloat16() for _ in range(3)]
    b = torch.zeros(E, device="cuda")
    off = torch.arange(M + 1, device="cuda") * T // M
    ws = eqb.EqbWorkspace(E)

    def outputs():
        return (torch.empty(T, K, dtype=torch.int32, device="cuda"), torch.empty(T, device="cuda"),
                torch.zeros(M, E, dtype=torch.int32, device="cuda"), torch.empty(E, device="cuda"))
    want = []
    for z in zs:
        o = outputs()
        eqb.eqb_layer_forward(z, b, K, off, ws, *o)
        want.append(o)
    got = [outputs() for _ in range(20) for _ in zs]
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        torch.cuda._sleep(5_000_000)  # the calls queue up behind it
    for i, o in enumerate(got):
        eqb.eqb_layer_forward(zs[i % 3], b, K, off, ws, *o, stream=st)
    torch.cuda.synchronize()
    assert ws.err.item() == 0
    for i, o in enumerate(got):
        assert all(torch.equal(x, y) for x, y in zip(o, want[i % 3]))
