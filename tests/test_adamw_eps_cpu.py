"""eqb_adamw_step's eps: refused where it is not a normal number in fp32.
Nothing is launched (no gradient is given), so no GPU is needed."""
import pytest

import paper_2609_28053_gb300 as eqb
from paper_2609_28053_gb300 import _lib

INVALID = 1


def step(eps):
    t = (_lib.AdamwTensor * 1)()
    t[0].n = 10
    return eqb.load().eqb_adamw_step(t, 1, 32, 1e-3, 1, 0.9, 0.95, eps, 0.1, None, None, None)


@pytest.mark.parametrize("eps", [1e-46, 1e-45, 1e-40, 1.17549e-38, 3.5e38, 1e300, 0.0, -1e-8, float("nan"), float("inf")])
def test_refused(eps):
    assert step(eps) == INVALID


@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-30, 1e-8, 1.0, 1e30])
def test_taken(eps):
    assert step(eps) == 0
