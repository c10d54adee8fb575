"""Orthogonalised updates over the whole range of fp32: G as small or as large as its type holds, on both sides of the sizes at
which the sums of squares leave the range and are taken again.

Bar.  The header's, which a power of two in front of G does not change: 1e-3 of the result's norm for independent elements, and for
small matrices of equal rows; 4e-3 where singular values fall off, and for a handful of rows in the tile kernels.  The reference takes G as
it is, denormals among its elements included.
"""
import pytest
import torch

from paper_1605_04711_b200 import twn
from _gpu_util import workspace
from test_gpu_orthogonalize import _exact, _normal, _run

pytestmark = pytest.mark.gpu

F, B = torch.float32, torch.bfloat16
BAR = 1e-3


def _near(G, O, steps=5, eps=1e-7, bar=BAR):
    want = _exact(G, steps, eps)
    assert bool(O.isfinite().all())
    assert float((O.double() - want).norm()) <= (bar + (2.0 ** -8 if O.dtype == B else 0.0)) * float(want.norm())


def _matrix(kind, rows, cols):
    """Of norm 1, in 64 bits."""
    G = _normal(rows + cols, rows, cols).double()
    if kind == "equal":                          # every row the same
        G = G[:1].repeat(rows, 1)
    elif kind == "one":                          # one row that counts, the others near nothing
        G[1:] *= 1e-4
    return G / G.norm()


@pytest.mark.parametrize("rows,cols,kind", [(1, 300, "any"), (1, 8192, "any"), (4, 300, "equal"), (4, 300, "any"), (10, 300, "equal"), (47, 500, "equal"), (47, 500, "any"),
                                            (128, 400, "equal"), (128, 8192, "any"), (128, 300, "one"), (300, 4, "equal"), (900, 100, "any")])
def test_every_decade_of_small_matrices(rows, cols, kind):
    G = _matrix(kind, rows, cols)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for k in range(-28, 39):
        # the last power leaves the largest element inside fp32
        g = (G * (10.0 ** k if k < 38 else 3e38 / float(G.abs().max()) / 1.01)).float()
        _near(g, _run([g], eps=1e-30, status=status)[0], eps=1e-30, bar=4e-3 if kind == "one" else BAR)
    assert twn.read_status(status) == 0


@pytest.mark.parametrize("gt", [F, B])
@pytest.mark.parametrize("rows,cols,kind", [(1, 64, "any"), (4, 64, "equal"), (64, 576, "any"), (128, 8192, "any"), (700, 20, "one")])
def test_both_sides_of_where_the_sums_are_taken_again(rows, cols, kind, gt):
    G = _matrix(kind, rows, cols)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for k in [*range(-60, -24), *range(44, 68)]:
        for scale in (2.0 ** k, 1.37 * 2.0 ** k):
            g = (G * scale).to(gt)
            _near(g, _run([g], eps=1e-30, status=status)[0], eps=1e-30, bar=4e-3 if kind == "one" else BAR)
    assert twn.read_status(status) == 0


@pytest.mark.parametrize("look", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 300), (64, 70), (300, 4), (200, 300)])
def test_a_momentum_that_dies_away(look, rows, cols):
    """Gradients that have stopped: V passes through every size on its way down.  Every step moves W by at most lr s |O|."""
    W, dW, V = _normal(1, rows, cols), torch.zeros(rows, cols, device="cuda"), _normal(2, rows, cols)
    V *= 1e-9 / float(V.norm())
    status, stats = torch.zeros(1, dtype=torch.int32, device="cuda"), twn.new_stats()
    ws = workspace(twn.muon_workspace_bytes([(rows, cols)]))
    s = max(1.0, rows / cols) ** 0.5
    mu = torch.tensor(0.95, dtype=F, device="cuda")
    for step in range(100):
        w, v = W.clone(), (V * mu)
        twn.muon_update_batch([(W, dW, V, rows, cols, stats)], 0.02, 0.95, 0.0, look, 5, 1e-30, 0.7, ws, status)
        assert torch.equal(V, v)
        # singular values of O are at most 1.21; a rounding of W on top
        assert float((W - w).double().norm()) <= 0.02 * s * 1.25 * min(rows, cols) ** 0.5 + 2.0 ** -24 * float(W.double().norm())
    assert twn.read_status(status) == 0 and twn.stats_to_host(stats)["status"] == 0
