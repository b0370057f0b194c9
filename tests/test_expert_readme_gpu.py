"""The experts' sequence of the README as it is written there, with lists that are cut
short, so that there are rows of no expert: memory that nobody has written must not
reach an error flag or a result."""
import functools
import re
from pathlib import Path

import pytest
import torch

import expert_reference as ref
import paper_2609_28053_gb300 as eqb

pytestmark = pytest.mark.gpu


class Flagged:
    """The package, each call that has an error flag with this one."""

    def __init__(self, err):
        self.err = err

    def __getattr__(self, name):
        call = getattr(eqb, name)
        has = name in ("eqb_gate_topk", "eqb_quant_rows", "eqb_quant_cols", "eqb_quant_blocks", "eqb_expert_matmul", "eqb_expert_wgrad")
        return functools.partial(call, err_flag=self.err) if has else call


class Poisoned:
    """torch, with NaN in what is made without values."""

    def __getattr__(self, name):
        made = getattr(torch, name)
        if name not in ("empty", "empty_like"):
            return made
        return lambda *a, **kw: made(*a, **kw).fill_(torch.nan)


def sequence():
    text = (Path(__file__).resolve().parent.parent / "README.md").read_text()
    return re.search(r"### The experts behind the router\n\n```python\n(.*?)```", text, re.S).group(1)


def test_the_sequence_with_rows_of_no_expert():
    T, n, d, E, K = 300, 144, 256, 16, 4
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(T, E, generator=g, device="cuda").bfloat16()
    z[::3] = -torch.inf      # all experts closed
    z[1::3, 2:] = -torch.inf  # all but two
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    at = {"torch": Poisoned(), "eqb": Flagged(err), "n": n, "d": d, "E": E, "K": K, "b": torch.zeros(E, device="cuda"), "z": z,
          "x": torch.randn(T, d, generator=g, device="cuda").bfloat16(), "dy": torch.randn(T, n, generator=g, device="cuda").bfloat16()}
    exec(sequence(), at)
    torch.cuda.synchronize()
    assert err.item() == 0
    assert int(at["offsets"][E]) < T * K
    for name in ("y", "dx", "dW", "dz", "dw"):
        assert torch.isfinite(at[name]).all(), name
    assert not at["dx"][::3].any() and not at["y"][::3].any()


def test_rows_that_are_none_can_be_left_out():
    """Sorted rows with a list of one entry each, -1 for the rows of no expert: those are neither read nor written."""
    T, n, E, K = 200, 272, 8, 4
    g = torch.Generator().manual_seed(2)
    idx = torch.randint(-1, E, (T, K), generator=g, dtype=torch.int32)
    offsets, _, slot, entry = (t.cuda() for t in eqb.eqb_expert_rows(idx.cuda(), E))
    x = torch.randn(T * K, n, generator=g).bfloat16().cuda()
    x[int(offsets[E]):] = torch.nan
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    own = torch.where(entry >= 0, torch.arange(T * K, device="cuda"), -1).int().view(-1, 1)
    q, s = torch.full((T * K, n), 1.0, device="cuda").to(torch.float8_e4m3fn), torch.full((T * K, 3), -3.0, device="cuda")
    eqb.eqb_quant_rows(x, own, q=q, scale=s, err_flag=err)
    assert err.item() == 0
    R = int(offsets[E])
    assert (s[R:] == -3.0).all() and (q[R:].float() == 1.0).all()
    want, ws = eqb.eqb_quant_rows(x[:R].contiguous())
    assert torch.equal(q[:R].view(torch.uint8), want.view(torch.uint8)) and torch.equal(s[:R], ws)
    eqb.eqb_quant_rows(x, err_flag=err)  # every row is read
    assert err.item() == 4
