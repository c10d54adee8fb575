"""SiLU of group norm where z is far below zero: z exp(z) and its slope, as far as fp32 has such numbers."""
import numpy as np
import pytest
import torch

from test_gpu_group_norm import F32, K, U, bwd, fwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(2, 300, 64, 8), (2, 90000, 24, 3), (3, 129, 7, 7)], ids=str)
def test_values_and_slopes(shape):
    B, HW, C, G = shape
    g = torch.Generator(device="cuda").manual_seed(5)
    X, dY = torch.randn(B * HW * C, device="cuda", generator=g), torch.rand(B * HW * C, device="cuda", generator=g) + 0.5
    gamma = torch.full((C,), 0.25, device="cuda")
    # channels around -20 to -84: |z - beta| is at most 0.25 times 6, so that none is below -87, where fp32 has no exp(z) of all its digits
    beta = torch.linspace(-20.0, -84.0, C, device="cuda")
    mean, rstd = torch.empty(B * G, device="cuda"), torch.empty(B * G, device="cuda")
    Y, dX = torch.empty_like(X), torch.empty_like(X)
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    fwd(X, C, B, HW, C, G, gamma, beta, "silu", Y, C, mean, rstd)
    bwd(dY, C, X, C, B, HW, C, G, gamma, beta, mean, rstd, "silu", dX, C, dgamma, dbeta)
    x = X.double().view(B, HW, G, C // G)
    xh = (x - mean.double().view(B, 1, G, 1)) * rstd.double().view(B, 1, G, 1)
    z = (xh.reshape(B, HW, C) * gamma.double() + beta.double())
    f = torch.sigmoid(z)
    # an error of z of K of its terms goes into exp(z) as it is; what the exponential, the sum and the quotient lose is K again
    e = K * (xh.abs().reshape(B, HW, C) * gamma.double() + 2.0 * z.abs()) + K
    y = z * f
    assert bool(((Y.double().view(B, HW, C) - y).abs() <= e * y.abs() + 1e-37).all())
    dz = dY.double().view(B, HW, C) * f * (1.0 + z * (1.0 - f))
    assert bool(((dbeta.double() - dz.sum((0, 1))).abs() <= (e * dz.abs()).sum((0, 1)) + 1e-37).all())


def test_below_all_numbers():
    """z of -100 to -1e30 and -infinity: next to nothing, no NaN."""
    C, HW = 32, 64
    X = torch.linspace(-3, 3, HW * C, device="cuda")
    Y, dX = torch.empty_like(X), torch.empty_like(X)
    mean, rstd = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    for beta in (-100.0, -1e4, -1e30, -float("inf")):
        gamma, b = torch.ones(C, device="cuda"), torch.full((C,), beta, device="cuda")
        dbeta = torch.empty(C, device="cuda")
        fwd(X, C, 1, HW, C, 4, gamma, b, "silu", Y, C, mean, rstd)
        bwd(torch.ones_like(X), C, X, C, 1, HW, C, 4, gamma, b, mean, rstd, "silu", dX, C, None, dbeta)
        for t in (Y, dX, dbeta):
            assert float(t.abs().max()) <= 1e-33
