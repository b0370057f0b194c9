"""Host-side refusals of the experts' entry points: nothing is launched, so no GPU is needed."""
import ctypes

import pytest
import torch

import paper_2609_28053_gb300 as eqb

INVALID, UNSUPPORTED = 1, 2
FAKE = ctypes.c_void_p(0x10000)
OFF2 = ctypes.c_void_p(0x10002)
OFF4 = ctypes.c_void_p(0x10004)
OFF16 = ctypes.c_void_p(0x10010)
NULL = None
HUGE = 2 ** 31


@pytest.fixture(scope="module")
def lib():
    return eqb.load()


def test_gate_refuses(lib):
    def call(z=FAKE, b=FAKE, T=100, E=64, K=4, groups=1, top=1, two=0, score=1, renorm=1, scale=1.0, mask=NULL, idx=FAKE, w=FAKE,
             err=NULL):
        return lib.eqb_gate_topk(z, 0, b, T, E, K, groups, top, two, score, renorm, scale, mask, idx, w, err, NULL)

    assert call(E=60) == UNSUPPORTED and call(E=1032) == UNSUPPORTED
    assert call(K=0) == INVALID and call(K=64) == INVALID and call(K=32) == UNSUPPORTED
    assert call(T=-1) == INVALID and call(T=HUGE) == UNSUPPORTED
    assert call(groups=0) == INVALID and call(groups=5) == INVALID and call(groups=8, top=0) == INVALID
    assert call(groups=8, top=9) == INVALID and call(groups=64, top=64) == UNSUPPORTED
    assert call(groups=32, top=1, K=4) == INVALID  # a group of two has no four experts
    assert call(score=2) == INVALID and call(score=-1) == INVALID
    assert call(scale=float("nan")) == INVALID and call(scale=1e39) == INVALID
    assert call(z=NULL) == INVALID and call(idx=NULL) == INVALID
    assert call(z=OFF4) == INVALID and call(b=OFF2) == INVALID and call(idx=OFF2) == INVALID and call(w=OFF2) == INVALID
    assert call(T=0, z=NULL, idx=NULL, w=NULL, b=NULL) == 0


def test_gate_grad_refuses(lib):
    def call(z=FAKE, idx=FAKE, gw=FAKE, T=100, E=64, K=4, score=1, renorm=1, scale=1.0, gi=NULL, go=FAKE, bf16=0):
        return lib.eqb_gate_grad(z, 0, idx, gw, T, E, K, score, renorm, scale, gi, go, bf16, NULL)

    assert call(E=60) == UNSUPPORTED and call(E=1032) == UNSUPPORTED and call(K=64) == INVALID and call(K=32) == UNSUPPORTED
    assert call(T=-1) == INVALID and call(T=HUGE) == UNSUPPORTED and call(score=3) == INVALID
    assert call(scale=float("inf")) == INVALID
    for name in ("z", "idx", "gw", "go"):
        assert call(**{name: NULL}) == INVALID
        assert call(**{name: OFF2}) == INVALID
    assert call(gi=OFF4) == INVALID and call(go=OFF4) == INVALID
    assert call(gi=FAKE, bf16=1) == INVALID  # fp32 in, bf16 out, one buffer
    assert call(T=0, z=NULL, idx=NULL, gw=NULL, go=NULL) == 0


def test_rows_refuses(lib):
    ws = lib.eqb_expert_rows_workspace_bytes(65536, 8, 128)
    assert ws > 0 and lib.eqb_expert_rows_workspace_bytes(64, 8, 256) == 0
    assert lib.eqb_expert_rows_workspace_bytes(-1, 8, 256) == 0

    def call(idx=FAKE, T=65536, K=8, E=128, off=FAKE, blk=FAKE, slot=FAKE, entry=FAKE, w=FAKE, wb=ws):
        return lib.eqb_expert_rows(idx, T, K, E, off, blk, slot, entry, w, wb, NULL)

    assert call(T=-1) == INVALID and call(K=0) == INVALID and call(E=0) == INVALID
    assert call(K=1025) == UNSUPPORTED and call(E=1025) == UNSUPPORTED and call(T=2 ** 28) == UNSUPPORTED
    assert call(T=2 ** 62, K=4) == UNSUPPORTED
    for name in ("idx", "off", "blk", "slot", "entry"):
        assert call(**{name: NULL}) == INVALID
        assert call(**{name: OFF2}) == INVALID
    assert call(w=NULL) == INVALID and call(wb=ws - 1) == INVALID and call(w=OFF4) == INVALID
    assert call(T=0, off=NULL) == INVALID


def test_max_blocks(lib):
    assert lib.eqb_expert_max_blocks(0, 8) == 0
    assert lib.eqb_expert_max_blocks(1, 8) == 1
    assert lib.eqb_expert_max_blocks(8, 8) == 8
    assert lib.eqb_expert_max_blocks(256, 128) == 129  # 127 experts with one row, one with 129
    assert lib.eqb_expert_max_blocks(1000, 1) == 8
    assert lib.eqb_expert_max_blocks(-1, 8) == -1 and lib.eqb_expert_max_blocks(8, 0) == -1
    for R in range(0, 40):  # all ways of cutting few rows
        for E in (1, 2, 3):
            cuts = [(R - i - j, i, j) for i in range(R + 1) for j in range(R + 1 - i)] if E == 3 else \
                [(R - i, i) for i in range(R + 1)] if E == 2 else [(R,)]
            assert lib.eqb_expert_max_blocks(R * 8, E) >= max(sum((8 * n + 127) // 128 for n in c) for c in cuts)


def test_quant_refuses(lib):
    def rows(x=FAKE, T=100, d=256, slot=FAKE, K=4, q=FAKE, s=FAKE):
        return lib.eqb_quant_rows(x, T, d, slot, K, q, s, NULL, NULL)

    assert rows(d=0) == INVALID and rows(d=24) == UNSUPPORTED and rows(d=2 ** 20 + 16) == UNSUPPORTED
    assert rows(T=-1) == INVALID and rows(T=HUGE) == UNSUPPORTED and rows(T=2 ** 30) == UNSUPPORTED and rows(K=0) == INVALID
    for name in ("x", "q", "s"):
        assert rows(**{name: NULL}) == INVALID
    assert rows(x=OFF4) == INVALID and rows(q=OFF4) == INVALID and rows(s=OFF2) == INVALID and rows(slot=OFF2) == INVALID
    assert rows(T=0, x=NULL) == 0

    def cols(x=FAKE, T=100, c=256, entry=FAKE, R=400, K=4, off=FAKE, blk=FAKE, E=8, P=11, q=FAKE, s=FAKE):
        return lib.eqb_quant_cols(x, T, c, entry, R, K, off, blk, E, P, q, s, NULL, NULL)

    assert cols(c=0) == INVALID and cols(c=40) == UNSUPPORTED and cols(E=0) == INVALID and cols(E=1025) == UNSUPPORTED
    assert cols(T=-1) == INVALID and cols(R=-1) == INVALID and cols(R=HUGE) == UNSUPPORTED and cols(K=0) == INVALID
    assert cols(P=-1) == INVALID and cols(P=2 ** 24) == UNSUPPORTED
    assert cols(entry=NULL) == INVALID  # 400 rows of 100
    for name in ("x", "off", "blk", "q", "s"):
        assert cols(**{name: NULL}) == INVALID
    assert cols(x=OFF4) == INVALID and cols(q=OFF4) == INVALID and cols(s=OFF2) == INVALID and cols(off=OFF2) == INVALID
    assert cols(P=0, q=NULL, s=NULL) == 0 and cols(R=0) == 0

    def blocks(w=FAKE, E=4, n=256, d=128, q=FAKE, s=FAKE, qt=FAKE, st=FAKE):
        return lib.eqb_quant_blocks(w, 0, E, n, d, q, s, qt, st, NULL, NULL)

    assert blocks(n=0) == INVALID and blocks(n=8) == UNSUPPORTED and blocks(d=17) == UNSUPPORTED and blocks(E=-1) == INVALID
    assert blocks(E=1025) == UNSUPPORTED
    for name in ("w", "q", "s", "qt", "st"):
        assert blocks(**{name: NULL}) == INVALID
    assert blocks(w=OFF4) == INVALID and blocks(q=OFF4) == INVALID and blocks(qt=OFF4) == INVALID and blocks(s=OFF2) == INVALID
    assert blocks(E=0, w=NULL) == 0


def test_matmul_refuses(lib):
    def mm(q=FAKE, s=FAKE, w=FAKE, ws=FAKE, off=FAKE, R=100, n=256, d=128, E=4, out=FAKE):
        return lib.eqb_expert_matmul(q, s, w, ws, off, R, n, d, E, out, 0, NULL, NULL)

    assert mm(n=0) == INVALID and mm(d=-16) == INVALID and mm(n=24) == UNSUPPORTED and mm(d=8) == UNSUPPORTED
    assert mm(E=0) == INVALID and mm(E=1025) == UNSUPPORTED and mm(R=-1) == INVALID and mm(R=HUGE) == UNSUPPORTED
    for name in ("q", "s", "w", "ws", "off", "out"):
        assert mm(**{name: NULL}) == INVALID
        assert mm(**{name: OFF2}) == INVALID
    assert mm(out=OFF16) == INVALID and mm(q=OFF4) == INVALID and mm(w=OFF4) == INVALID
    assert mm(R=0, q=NULL, out=NULL) == 0

    def wg(a=FAKE, sa=FAKE, b=FAKE, sb=FAKE, blk=FAKE, P=5, n=256, d=128, E=4, dW=FAKE, add=0):
        return lib.eqb_expert_wgrad(a, sa, b, sb, blk, P, n, d, E, dW, add, NULL, NULL)

    assert wg(n=0) == INVALID and wg(d=40) == UNSUPPORTED and wg(E=0) == INVALID and wg(P=-1) == INVALID and wg(P=2 ** 24) == UNSUPPORTED
    for name in ("a", "sa", "b", "sb", "blk", "dW"):
        assert wg(**{name: NULL}) == INVALID
        assert wg(**{name: OFF2}) == INVALID
    assert wg(dW=OFF16) == INVALID and wg(sb=OFF4) == INVALID
    assert wg(P=0, add=1, a=NULL, sa=NULL, b=NULL, sb=NULL) == 0


def test_combine_refuses(lib):
    def fwd(rows=FAKE, slot=FAKE, w=FAKE, T=100, R=400, n=256, K=4, out=FAKE):
        return lib.eqb_expert_combine(rows, slot, w, T, R, n, K, out, NULL)

    def bwd(g=FAKE, rows=FAKE, slot=FAKE, w=FAKE, T=100, R=400, n=256, K=4, gr=FAKE, gw=FAKE):
        return lib.eqb_expert_combine_grad(g, rows, slot, w, T, R, n, K, gr, gw, NULL)

    for call in (fwd, bwd):
        assert call(n=0) == INVALID and call(n=24) == UNSUPPORTED and call(K=0) == INVALID and call(K=1025) == UNSUPPORTED
        assert call(T=-1) == INVALID and call(R=-1) == INVALID and call(T=HUGE) == UNSUPPORTED and call(R=HUGE) == UNSUPPORTED
        for name in ("rows", "slot"):
            assert call(**{name: NULL}) == INVALID
            assert call(**{name: OFF2}) == INVALID
        assert call(w=OFF2) == INVALID
        assert call(T=0, rows=NULL, slot=NULL) == 0
    assert fwd(out=NULL) == INVALID and fwd(out=OFF4) == INVALID
    assert bwd(g=NULL) == INVALID and bwd(gr=OFF4) == INVALID and bwd(gw=OFF2) == INVALID
    assert bwd(gr=NULL, gw=NULL) == 0


def test_bindings_refuse():
    z = torch.zeros(4, 16, dtype=torch.bfloat16)
    i32 = torch.zeros(4, 2, dtype=torch.int32)
    q = torch.zeros(16, 16, dtype=torch.float8_e4m3fn)
    off = torch.zeros(2, dtype=torch.int32)
    w3 = torch.zeros(1, 16, 16, dtype=torch.bfloat16)
    for call in (lambda: eqb.eqb_gate_topk(z, None, 2), lambda: eqb.eqb_gate_grad(z, i32, torch.zeros(4, 2)),
                 lambda: eqb.eqb_expert_rows(i32, 16), lambda: eqb.eqb_quant_rows(z), lambda: eqb.eqb_quant_cols(z, off, off),
                 lambda: eqb.eqb_quant_blocks(w3),
                 lambda: eqb.eqb_expert_matmul(q, torch.zeros(16, 1), q[None], torch.zeros(1, 1, 1), off),
                 lambda: eqb.eqb_expert_combine(z, i32), lambda: eqb.eqb_expert_combine_grad(z, z, i32)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="dimensions"):
        eqb.eqb_gate_topk(z[0], None, 2)
    with pytest.raises(ValueError, match="dimensions"):
        eqb.eqb_quant_blocks(z)
    with pytest.raises(TypeError):
        eqb.eqb_gate_topk(None, None, 2)
    with pytest.raises(TypeError):
        eqb.eqb_quant_rows(z.float())
