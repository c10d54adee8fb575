"""Gradients of group norm in columns of hundreds of pixels a thread."""
import pytest
import torch

from test_gpu_group_norm import BF16, U, bwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("HW,C", [(8000, 51), (4000, 102)])
def test_small_gradients_behind_a_large_one(HW, C):
    """The first pixels have gradients of 1, as many of them as a block of 256 threads has of rows; all others have 0.99 u, which a sum of 1 does not take up.  In runs of
    64 pixels a thread loses at most the 63 of the first run; the sums of the runs, of the threads and of the tiles behind it are 20 roundings."""
    B = 150
    V = 1 if C % 2 else 2
    rows = 256 // (C // V)
    dY = torch.full((B, HW, C), 0.9921875 * U, dtype=BF16, device="cuda")
    dY[:, :rows] = 1.0
    g = torch.Generator(device="cuda").manual_seed(1)
    X = torch.empty(B, HW, C, dtype=BF16, device="cuda").uniform_(1.0, 2.0, generator=g)
    X[:, :rows] = 1.0
    mean, rstd = torch.zeros(B, device="cuda"), torch.ones(B, device="cuda")
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    bwd(dY.view(-1), C, X.view(-1), C, B, HW, C, 1, None, None, mean, rstd, "none", None, C, dgamma, dbeta)
    for got, want in ((dbeta, dY.double().sum((0, 1))), (dgamma, (dY.double() * X.double()).sum((0, 1)))):
        assert float((got.double() / want - 1.0).abs().max()) <= 84 * U
