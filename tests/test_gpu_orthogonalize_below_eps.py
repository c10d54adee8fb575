"""Orthogonalised updates of matrices far below eps, which stay far below 1: X = G / eps keeps its digits, however small it is.

Bar.  The header's: 1e-3 of the result's norm for independent elements with five steps or fewer, or with as many steps past those
that only multiply by a = 3.4445; 4e-3 for a handful of rows in the tile kernels.  The reference takes G as it is, denormals among its
elements included.
"""
import pytest
import torch

from paper_1605_04711_b200 import twn
from test_gpu_orthogonalize import NS, _run
from test_gpu_orthogonalize_range import BAR, _matrix, _near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(1, 300), (60, 300), (300, 60), (128, 8192), (64, 576), (200, 300), (1000, 513), (2820, 3100), (130, 9000)])
@pytest.mark.parametrize("norm,eps,steps", [(1e-7, 1e-7, 5), (1e-8, 1e-7, 5), (3e-10, 1e-7, 1), (1e-11, 1e-7, 5), (1e-13, 1e-7, 5), (1e-20, 1e-7, 5), (1e-30, 1e-7, 5), (1e-36, 1e-7, 2),
                                            (1e-13, 1e-7, 16), (1e-5, 1.0, 9), (1e-4, 1e5, 18), (1.0, 1e20, 5), (1e-30, 1e-30, 5), (1e-33, 1e-30, 7), (1e30, 1e30, 5), (1e10, 1e30, 3)])
def test_far_below_eps(rows, cols, norm, eps, steps):
    """Five steps past where the first singular values reach 1, at most, as the bar asks."""
    G = (_matrix("any", rows, cols) * norm).float()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    O = _run([G], steps=steps, eps=eps, status=status)[0]
    _near(G, O, steps, eps, 4e-3 if min(rows, cols) < 64 and steps > 5 else BAR)
    assert twn.read_status(status) == 0
    if norm / eps * NS[0] ** steps < 2.0 ** -12:
        # linear up to 2^-24: O is a multiple of G
        assert float((O.double() - G.double() * (NS[0] ** steps / eps)).norm()) <= 1e-5 * float(O.double().norm())
