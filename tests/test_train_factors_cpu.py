"""Factors of the training calls that are finite in fp64 and not in fp32 are
refused, and nothing is launched."""
import ctypes

import pytest

import paper_2609_28053_gb300 as eqb
from paper_2609_28053_gb300 import _lib

INVALID = 1
FAKE = ctypes.c_void_p(0x10000)


@pytest.mark.parametrize("alpha,zeta", [(1e39, 0.0), (-1e39, 0.0), (1e300, 0.0), (0.1, 1e39), (0.1, -1e300), (0.1, 3e38)])
def test_balance_loss_refuses(alpha, zeta):
    # 3e38: the gradient takes 2 zeta
    assert eqb.load().eqb_balance_loss(FAKE, 0, FAKE, 100, 64, 4, FAKE, 2, None, 0, alpha, zeta, None, FAKE, 0, None, FAKE, None,
                                       None, None, 0, None, None) == INVALID


def adamw(lr, wd, step=1, b1=0.9):
    t = (_lib.AdamwTensor * 1)()
    t[0].n = 10  # no gradient: nothing to do
    return eqb.load().eqb_adamw_step(t, 1, 32, lr, step, b1, 0.95, 1e-8, wd, None, None, None)


@pytest.mark.parametrize("lr,wd", [(1e39, 0.0), (1e300, 0.0), (1e38, 0.0), (1e-3, 1e300), (1e30, 1e30)])
def test_adamw_refuses(lr, wd):
    assert adamw(lr, wd) == INVALID  # 1e38 / (1 - 0.9) is beyond fp32


def test_adamw_takes():
    assert adamw(1e30, 1e-3) == 0 and adamw(0.0, 1e30) == 0 and adamw(1e38, 0.0, step=1, b1=0.0) == 0
