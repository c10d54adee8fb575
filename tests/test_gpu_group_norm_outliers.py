"""Mean and variance of groups whose first values are far from all others.

Bounds.  A difference from what it is taken from is off by half a step of itself, u, and so is every addition of a thread; a thread has some dozens of those one after the other, of random
sign.  With K = 40 u as elsewhere: the mean is off by K times the mean size of the values at most, 1/deviation by K of itself."""
import pytest
import torch

from test_gpu_group_norm import EPS, K, fwd

pytestmark = pytest.mark.gpu


def _run(X, B, HW, C, G):
    mean, rstd = torch.empty(B * G, device="cuda"), torch.empty(B * G, device="cuda")
    Y = torch.empty_like(X)
    fwd(X, C, B, HW, C, G, None, None, "none", Y, C, mean, rstd)
    return Y, mean.double().view(B, G), rstd.double().view(B, G)


def _check(X, mean, rstd, B, HW, C, G, images):
    for b in images:
        x = X.view(B, HW, G, C // G)[b].double()
        want = x.mean((0, 2))
        var = (x - want[None, :, None]).square().mean((0, 2))
        off = (mean[b] - want).abs() / (K * x.abs().mean((0, 2)))
        assert float(off.max()) <= 1.0, ("mean", b, float(off.max()))
        off = (rstd[b] * (var + EPS).sqrt() - 1.0).abs() / K
        assert float(off.max()) <= 1.0, ("rstd", b, float(off.max()))


@pytest.mark.parametrize("shape", [(2, 500, 64, 8), (1, 2000, 32, 4), (1, 90000, 24, 3), (2, 300, 24, 8), (3, 129, 7, 7), (2, 333, 150, 50)], ids=str)
def test_the_first_pixel(shape):
    """The first value of every group, and the whole first pixel, at 6e4: few pixels a thread."""
    B, HW, C, G = shape
    g = torch.Generator(device="cuda").manual_seed(1)
    for whole in (False, True):
        X = torch.randn(B, HW, C, device="cuda", generator=g)
        X[:, 0, ::1 if whole else C // G] = 6e4
        X = X.view(-1)
        Y, mean, rstd = _run(X, B, HW, C, G)
        _check(X, mean, rstd, B, HW, C, G, range(B))
