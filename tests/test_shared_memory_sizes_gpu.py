"""Calls whose shared memory lies about what a launch has without asking for more, each
as the first of a process: what an earlier call asked for must not matter."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
TESTS = Path(__file__).resolve().parent

ROWS = """
import sys, torch
sys.path[:0] = [{root!r}, {tests!r}]
import expert_reference as ref
import paper_2609_28053_gb300 as eqb
E, T, K = {E}, {T}, 3
idx = torch.randint(-1, E, (T, K), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
got = eqb.eqb_expert_rows(idx.cuda(), E)
for g, w in zip(got, ref.rows(idx, E)):
    assert g.cpu().flatten().tolist() == w
"""


MAXVIO = """
import sys, torch
sys.path[:0] = [{root!r}, {tests!r}]
import paper_2609_28053_gb300 as eqb
M, E, K, n = {M}, 8, 2, 16
loads = torch.full((M, E), n * K // E, dtype=torch.int32)
loads[:, 3] += 2
loads[:, 5] -= 2
out = eqb.eqb_maxvio(loads.cuda(), (torch.arange(M + 1) * n).cuda(), K)
out = out[0] if isinstance(out, tuple) else out
assert (out.cpu() == 0.5).all(), out
"""


def alone(code, **sizes):
    code = code.format(root=str(TESTS.parent), tests=str(TESTS), **sizes)
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


@pytest.mark.parametrize("E", [645, 646, 647])
@pytest.mark.parametrize("T", [50, 5000])
def test_rows_as_the_first_call(E, T):
    alone(ROWS, E=E, T=T)


@pytest.mark.parametrize("M", [6128, 6129, 6144, 6145])
def test_maxvio_as_the_first_call(M):
    alone(MAXVIO, M=M)
