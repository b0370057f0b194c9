"""eqb_expert_rows: whole numbers, equal to a plain sort."""
import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb
from gpu_harness import Guarded

pytestmark = pytest.mark.gpu


def run(idx, E, **kw):
    T, K = idx.shape
    out = [Guarded((E + 1,), torch.int32, fill=-9), Guarded((E + 1,), torch.int32, fill=-9), Guarded((T, K), torch.int32, fill=-9),
           Guarded((T * K,), torch.int32, fill=-9)]
    n = eqb.eqb_expert_rows_workspace_bytes(T, K, E)
    ws = torch.full((max(n, 1),), 0xff, dtype=torch.uint8, device="cuda")
    eqb.eqb_expert_rows(idx.cuda(), E, *[o.view for o in out], workspace=ws, **kw)
    torch.cuda.synchronize()
    assert all(o.intact() for o in out)
    return [o.view.cpu() for o in out]


def check(idx, E):
    got = run(idx, E)
    for g, w in zip(got, ref.rows(idx, E)):
        assert g.flatten().tolist() == w


def lists(T, E, K, seed, drop=0.0, skew=False):
    g = torch.Generator().manual_seed(seed)
    idx = torch.randint(0, E, (T, K), generator=g, dtype=torch.int32)  # an expert twice, too
    if skew:
        idx = (idx.float() ** 2 / E).int()
    idx[torch.rand(T, K, generator=g) < drop] = -1
    return idx


@pytest.mark.parametrize("T,E,K", [(1, 1, 1), (1, 8, 2), (3, 256, 8), (64, 256, 8), (511, 128, 8), (512, 128, 8), (513, 7, 8), (100, 1024, 31),
                                   (4096, 3, 1), (4097, 3, 1), (5000, 1000, 6), (20000, 128, 8), (65536, 1024, 2), (9, 5, 1000),
                                   (200000, 64, 3)])
@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_rows(T, E, K, drop):
    check(lists(T, E, K, T + E, drop, skew=T % 2 == 1), E)


def test_one_expert_has_all_and_none_has_any():
    check(torch.full((3000, 8), 5, dtype=torch.int32), 16)
    check(torch.full((3000, 8), -1, dtype=torch.int32), 16)
    check(torch.full((40, 8), 16, dtype=torch.int32), 16)
    check(torch.tensor([[2 ** 31 - 1, -2 ** 31, 3, 3]], dtype=torch.int32), 4)


def test_no_tokens():
    off, blk, slot, entry = eqb.eqb_expert_rows(torch.empty(0, 8, dtype=torch.int32, device="cuda"), 16)
    assert not off.any() and not blk.any() and off.shape == (17,) and slot.shape == (0, 8) and entry.shape == (0,)


def test_two_graphs_share_a_workspace():
    a, b = lists(9000, 128, 8, 1).cuda(), lists(9000, 128, 8, 2).cuda()
    ws = torch.empty(eqb.eqb_expert_rows_workspace_bytes(9000, 8, 128), dtype=torch.uint8, device="cuda")
    outs, graphs = [], []
    for x in (a, b):
        out = eqb.eqb_expert_rows(x, 128, workspace=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            eqb.eqb_expert_rows(x, 128, *out, workspace=ws)
        outs.append(out)
        graphs.append(graph)
    for out in outs:
        for t in out:
            t.fill_(-5)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for x, out in zip((a, b), outs):
        for g, w in zip(out, ref.rows(x.cpu(), 128)):
            assert g.cpu().flatten().tolist() == w


def test_made_memory_belongs_to_the_stream():
    idx = lists(30000, 64, 8, 3).cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = eqb.eqb_expert_rows(idx, 64, stream=s)
    s.synchronize()
    for g, w in zip(got, ref.rows(idx.cpu(), 64)):
        assert g.cpu().flatten().tolist() == w
