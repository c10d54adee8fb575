"""twn_layer_norm_fwd and twn_layer_norm_bwd refuse, on the host, outputs that lie over what else a call reads or writes, and serve rows that
lie between each other's."""
import ctypes as C

import pytest

import test_layer_norm_checks as checks
from test_layer_norm_checks import BF16, F32, INVALID, bwd, fwd, lib  # noqa: F401

BASE = 1 << 30                   # never dereferenced
SIZE = {F32: 4, BF16: 2}
STEP = 1 << 24


@pytest.fixture(autouse=True)
def _addresses_are_made_up():
    """A call that is served goes on to the device: these run only where there is none."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")


def _served(code):
    return code not in (INVALID, checks.MISALIGNED, checks.WORKSPACE, checks.TOO_LARGE, 0)


def _fwd(lib, **kw):
    at = {"X": BASE, "Y": BASE + STEP, "gamma": BASE + 2 * STEP, "beta": BASE + 3 * STEP, "mean": BASE + 4 * STEP, "rstd": BASE + 5 * STEP}
    return fwd(lib, **{**at, **kw})


def _bwd(lib, M=4, Cc=64, **kw):
    names = ["dY", "X", "gamma", "mean", "rstd", "dX", "dgamma", "dbeta", "ws"]
    at = {n: BASE + i * STEP for i, n in enumerate(names)}
    size = lib.twn_layer_norm_bwd_workspace_bytes(C.c_int64(M), C.c_int64(Cc))
    return bwd(lib, **{**at, "M": M, "Cc": Cc, "bytes_": size, **kw})


ROW = 64 * 4
FORWARD_REFUSED = [
    {"Y": BASE, "yt": BF16},                                     # X's place in another type
    {"Y": BASE, "yt": BF16, "ldy": 128},                         # row by row in X's rows
    {"Y": BASE, "ldy": 80},                                      # another pitch
    {"Y": BASE + ROW}, {"Y": BASE - ROW}, {"Y": BASE + 4}, {"Y": BASE + 4 * ROW - 4}, {"Y": BASE - 4 * ROW + 4},
    {"Y": BASE + 252, "ldx": 128, "ldy": 128}, {"Y": BASE + 3 * 512 + 252, "ldx": 128, "ldy": 128},
    {"Y": BASE + 256, "ldx": 127, "ldy": 128, "M": 1000},        # rows of two pitches that meet from the first or the second on
    {"mean": BASE + 40}, {"rstd": BASE + 4 * ROW - 4}, {"mean": BASE + STEP + 8}, {"mean": BASE + 5 * STEP}, {"mean": BASE + 5 * STEP + 12},
    {"mean": BASE + 2 * STEP + 16}, {"rstd": BASE + 3 * STEP - 12}, {"gamma": BASE + STEP + 4}, {"beta": BASE + STEP + 4 * ROW - 4},
]
FORWARD_SERVED = [
    {}, {"Y": BASE}, {"Y": BASE, "xt": BF16, "yt": BF16}, {"Y": BASE, "ldx": 70, "ldy": 70}, {"Y": BASE, "M": 1, "ldx": 64, "ldy": 99}, {"Y": BASE + 4 * ROW}, {"Y": BASE - 4 * ROW},
    {"Y": BASE + 256, "ldx": 128, "ldy": 128}, {"Y": BASE - 256, "ldx": 128, "ldy": 128},          # two halves of the rows of one buffer
    {"Y": BASE + 256, "yt": BF16, "ldx": 128, "ldy": 256}, {"Y": BASE + 384, "yt": BF16, "ldx": 128, "ldy": 256},
    {"X": BASE, "Y": BASE + 256, "ldx": 128, "ldy": 256, "M": 2},                                    # rows of 512 and of 1024 bytes that pass each other
    {"mean": BASE + 256, "ldx": 128, "M": 4}, {"gamma": BASE, "beta": BASE}, {"mean": 0, "rstd": 0}, {"gamma": 0, "beta": 0},
    {"mean": BASE + 4 * ROW, "rstd": BASE + 4 * ROW + 16}, {"Y": BASE + 256, "ldx": 128, "ldy": 128, "M": 1 << 20, "gamma": 0, "beta": 0, "mean": 0, "rstd": 0},
]


@pytest.mark.parametrize("args", FORWARD_REFUSED)
def test_forward_refuses(lib, args):  # noqa: F811
    assert _fwd(lib, **args) == INVALID


@pytest.mark.parametrize("args", FORWARD_SERVED)
def test_forward_serves(lib, args):  # noqa: F811
    assert _served(_fwd(lib, **args))


BACKWARD_REFUSED = [
    {"dX": BASE, "ot": BF16}, {"dX": BASE, "lddx": 70}, {"dX": BASE + STEP, "lddx": 65}, {"dX": BASE + ROW}, {"dX": BASE + STEP - 4},
    {"dX": BASE, "residual": BASE + 4}, {"residual": BASE + 5 * STEP + 4}, {"dgamma": BASE + 7 * STEP}, {"dgamma": BASE + 7 * STEP + 252}, {"dbeta": BASE + 2 * STEP},
    {"dgamma": BASE + 5 * STEP + 8}, {"dbeta": BASE + 3 * STEP - 248}, {"ws": BASE}, {"ws": BASE + 6 * STEP}, {"dX": BASE + 8 * STEP + 256}, {"ws": BASE + 2 * STEP - 1024},
]
BACKWARD_SERVED = [
    {}, {"dX": BASE}, {"dX": BASE + STEP}, {"dX": BASE, "X": BASE}, {"residual": BASE + 5 * STEP}, {"residual": BASE + 20 * STEP}, {"dX": BASE, "residual": BASE},
    {"dX": BASE + 256, "lddx": 128, "lddy": 128}, {"dX": 0}, {"dgamma": 0}, {"dbeta": 0, "dX": 0}, {"mean": BASE + 3 * STEP, "rstd": BASE + 3 * STEP}, {"gamma": 0},
    {"dbeta": BASE + 6 * STEP + 256}, {"M": 0, "dX": BASE + 6 * STEP},
]


@pytest.mark.parametrize("args", BACKWARD_REFUSED)
def test_backward_refuses(lib, args):  # noqa: F811
    assert _bwd(lib, **args) == INVALID


@pytest.mark.parametrize("args", BACKWARD_SERVED)
def test_backward_serves(lib, args):  # noqa: F811
    assert _served(_bwd(lib, **args))
