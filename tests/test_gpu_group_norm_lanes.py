"""Group norm with SiLU where a vector's channels are of different groups: what is not finite in one of them stays there."""
import pytest
import torch

from test_gpu_group_norm import BF16, F32, bwd, fwd

pytestmark = pytest.mark.gpu

# groups of an odd number of channels in vectors of eight (four in fp32) and of two; the last two are read twice
SHAPES = [(3, 333, 16, 16), (2, 300, 24, 8), (2, 600, 44, 4), (2, 77, 66, 22), (2, 300, 64, 64), (2, 90000, 24, 8), (2, 90000, 44, 4)]
NAN, INF = float("nan"), float("inf")


def _both(X, dY, gamma, beta, act, B, HW, C, G):
    mean, rstd = torch.empty(B * G, device="cuda"), torch.empty(B * G, device="cuda")
    Y, dX = torch.empty_like(X), torch.empty_like(X)
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    fwd(X, C, B, HW, C, G, gamma, beta, act, Y, C, mean, rstd)
    bwd(dY, C, X, C, B, HW, C, G, gamma, beta, mean, rstd, act, dX, C, dgamma, dbeta)
    return Y.view(B, HW, C), dX.view(B, HW, C), dgamma, dbeta


def _inputs(B, HW, C, dtype):
    g = torch.Generator(device="cuda").manual_seed(C + HW)
    X, dY = (torch.randn(B * HW * C, device="cuda", generator=g).to(dtype) for _ in range(2))
    return X, dY, 1.0 + 0.3 * torch.randn(C, device="cuda", generator=g), 0.3 * torch.randn(C, device="cuda", generator=g)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["silu", "relu"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_an_input(shape, act, dtype):
    """In the first or the last channel of a group: NaNs in that group of that image, the bits of a call without it everywhere else."""
    B, HW, C, G = shape
    Cg = C // G
    X, dY, gamma, beta = _inputs(B, HW, C, dtype)
    clean = _both(X, dY, gamma, beta, act, B, HW, C, G)
    assert all(bool(t.isfinite().all()) for t in clean)
    for bad, c in ((NAN, Cg), (INF, 2 * Cg - 1), (-INF, Cg)):
        x = X.clone()
        x.view(B, HW, C)[1, HW // 2, c] = bad
        got = _both(x, dY, gamma, beta, act, B, HW, C, G)
        for a, b in zip(clean[:2], got[:2]):
            assert bool(b[1, :, Cg:2 * Cg].isnan().all())
            b[1, :, Cg:2 * Cg] = a[1, :, Cg:2 * Cg]
            assert torch.equal(a, b)
        for a, b in zip(clean[2:], got[2:]):
            assert bool(b[Cg:2 * Cg].isnan().all())
            b[Cg:2 * Cg] = a[Cg:2 * Cg]
            assert torch.equal(a, b)


@pytest.mark.parametrize("which", ["gamma", "beta"])
@pytest.mark.parametrize("act", ["silu", "relu"])
@pytest.mark.parametrize("shape", SHAPES + [(2, 300, 64, 8), (2, 90000, 32, 1)], ids=str)
def test_a_parameter(shape, act, which):
    """NaN in one channel's gamma or beta: in Y, dgamma and dbeta that channel alone, in dX its group."""
    B, HW, C, G = shape
    Cg = C // G
    X, dY, gamma, beta = _inputs(B, HW, C, BF16)
    clean = _both(X, dY, gamma, beta, act, B, HW, C, G)
    for c in (Cg, 2 * Cg - 1) if G > 1 else (3, 4):
        p = {"gamma": gamma.clone(), "beta": beta.clone()}
        p[which][c] = NAN
        got = _both(X, dY, p["gamma"], p["beta"], act, B, HW, C, G)
        for k, (a, b) in enumerate(zip(clean, got)):
            own = slice(c // Cg * Cg, c // Cg * Cg + Cg) if k == 1 else slice(c, c + 1)
            assert bool(b[..., own].isnan().all())
            b[..., own] = a[..., own]
            assert torch.equal(a, b)


def test_one_gradient():
    """A NaN in dY: in dgamma and dbeta its channel alone, in dX its group of its image."""
    for B, HW, C, G in SHAPES:
        Cg = C // G
        X, dY, gamma, beta = _inputs(B, HW, C, BF16)
        clean = _both(X, dY, gamma, beta, "silu", B, HW, C, G)
        dy = dY.clone()
        dy.view(B, HW, C)[0, HW - 1, 2 * Cg - 1] = NAN
        got = _both(X, dy, gamma, beta, "silu", B, HW, C, G)
        assert torch.equal(clean[0], got[0])
        assert bool(got[1][0, :, Cg:2 * Cg].isnan().all())
        got[1][0, :, Cg:2 * Cg] = clean[1][0, :, Cg:2 * Cg]
        for a, b in zip(clean[2:], got[2:]):
            assert bool(b[2 * Cg - 1].isnan())
            b[2 * Cg - 1] = a[2 * Cg - 1]
        assert all(torch.equal(a, b) for a, b in zip(clean, got))
