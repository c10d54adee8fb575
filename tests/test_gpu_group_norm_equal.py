"""Group norm of groups whose values are all equal."""
import pytest
import torch

from test_gpu_group_norm import EPS, K, _backward64, _check_backward, bwd, fwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1, 100, 64, 8), (1, 90000, 24, 3), (2, 50, 7, 7), (160, 1000, 51, 1), (300, 20000, 50, 2), (2, 333, 150, 50)], ids=str)
@pytest.mark.parametrize("value", [3.7, -1e-3, 12345.678, 1e-30], ids=str)
def test_equal_values(shape, value):
    """The mean is the value, to the bit, and the variance 0: with eps = 0 1/deviation is infinite and Y NaN, as the formula has it."""
    B, HW, C, G = shape
    X = torch.full((B * HW * C,), value, device="cuda")
    mean, rstd = torch.empty(B * G, device="cuda"), torch.empty(B * G, device="cuda")
    Y = torch.empty_like(X)
    fwd(X, C, B, HW, C, G, None, None, "none", Y, C, mean, rstd)
    assert bool((Y == 0).all()) and bool((mean == X[0]).all())
    assert float((rstd.double() * EPS ** 0.5 - 1.0).abs().max()) <= K
    fwd(X, C, B, HW, C, G, None, None, "none", Y, C, mean, rstd, eps=0.0)
    assert bool(rstd.isinf().all()) and bool((mean == X[0]).all()) and bool(Y.isnan().all())


@pytest.mark.parametrize("shape", [(1, 100, 64, 8), (1, 90000, 24, 3), (2, 50, 7, 7), (2, 333, 150, 50)], ids=str)
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_groups_of_equal_values(shape, act):
    """xh is 0: dX is dz gamma / sqrt(eps) less its mean, dgamma is 0."""
    B, HW, C, G = shape
    g = torch.Generator(device="cuda").manual_seed(2)
    X, dY = torch.full((B * HW * C,), 3.7, device="cuda"), torch.randn(B * HW * C, device="cuda", generator=g)
    gamma, beta = 1.0 + 0.3 * torch.randn(C, device="cuda", generator=g), 0.3 * torch.randn(C, device="cuda", generator=g)
    mean, rstd = torch.full((B * G,), X[0].item(), device="cuda"), torch.full((B * G,), EPS ** -0.5, device="cuda")
    dX, dgamma, dbeta = torch.empty_like(X), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    bwd(dY, C, X, C, B, HW, C, G, gamma, beta, mean, rstd, act, dX, C, dgamma, dbeta)
    want = _backward64(dY.double(), X.double(), mean, rstd, gamma, beta, act, B, HW, G)
    # (what _backward64 allows for roundings of the differences, which are none here)
    assert bool((dgamma == 0).all())
    f = torch.sigmoid(beta.double()) if act == "silu" else None
    slope = {"none": 1.0, "relu": (beta > 0).double(), "silu": None if f is None else f * (1.0 + beta.double() * (1.0 - f))}[act]
    gz = (dY.double().view(B, HW, C) * slope * gamma.double()).view(B, HW, G, C // G)
    dx = (gz - gz.mean((1, 3), keepdim=True)) * rstd[0].double()
    off = (dX.double().view_as(dx) - dx).abs() / (rstd[0].double() * K * (gz.abs() + gz.abs().mean((1, 3), keepdim=True)) + 1e-30)
    assert float(off.max()) <= 1.0, float(off.max())
    _check_backward(want, None, dgamma, dbeta, B, HW, C, G)
