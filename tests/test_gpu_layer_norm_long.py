"""Layer norm of the longest rows and of the most rows, and with parameters on any boundary.

Bars, with u = 2^-24.  A sum over a row, whatever its length: eight additions of a vector, the rounding of a thread's total, five levels of
a tree, 32 warps one after the other and the product with a rounded 1 / C: k = 48 roundings of at most u sum|terms| each.
"""
import pytest
import torch

from paper_1605_04711_b200 import twn
from _gpu_util import workspace

pytestmark = pytest.mark.gpu

F, B = torch.float32, torch.bfloat16
U, K, EPS = 2.0 ** -24, 48, 1e-5
HALF = {F: U, B: 2.0 ** -8}
LENGTHS = [(5, 33001), (3, 65536), (3, 65537), (2, 1 << 20), (2, (1 << 22) + 3), (1, 1 << 26), (1, (1 << 27) + 8)]


def _randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("M,C", LENGTHS)
@pytest.mark.parametrize("dtype", [F, B])
def test_forward_of_long_rows(M, C, dtype):
    """Rows about 1.1 with a deviation of 0.05: an error of the mean shows twenty times."""
    x = (1.1 + 0.05 * _randn(C, M, C)).to(dtype)
    y, mean, rstd = torch.empty(M, C, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    twn.layer_norm_fwd(x, C, M, C, None, None, EPS, y, C, mean, rstd)
    for r in range(M):
        v = x[r].double()
        m = v.mean()
        d = v - m
        s = 1.0 / ((d * d).mean() + EPS).sqrt()
        e_mean = K * U * float(v.abs().mean())
        assert abs(float(mean[r]) - float(m)) <= e_mean
        # of the variance: k u of itself, two roundings of every difference, and the square of the mean's error
        rel = 0.5 * ((K + 6) * U + (e_mean * float(s)) ** 2) + 3 * U
        assert abs(float(rstd[r]) - float(s)) <= rel * float(s)
        want = d * s
        # x - mean is off by the mean's error and a rounding, then come the product and rstd
        bound = (e_mean + U * d.abs()) * float(s) + want.abs() * (rel + 2 * U)
        assert bool(((y[r].double() - want).abs() <= bound).all())


@pytest.mark.parametrize("M,C", LENGTHS)
@pytest.mark.parametrize("dtype", [F, B])
def test_backward_of_long_rows(M, C, dtype):
    """Gradients of one sign, so that their sums only grow."""
    x, dy = _randn(C, M, C).to(dtype), (0.7 + 0.1 * _randn(C + 1, M, C)).to(dtype)
    v = x.double()
    m = v.mean(1)
    mean, rstd = m.float(), (1.0 / ((v - m[:, None]).square().mean(1) + EPS).sqrt()).float()
    dx, dg, db = torch.empty(M, C, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = workspace(twn.layer_norm_bwd_workspace_bytes(M, C))
    ws.fill_(255)
    twn.layer_norm_bwd(dy, C, x, C, M, C, None, mean, rstd, dx, C, dg, db, ws)
    sums = torch.zeros(2, C, dtype=torch.float64, device="cuda")
    for r in range(M):
        g, s = dy[r].double(), float(rstd[r])
        xh = (v[r] - float(mean[r])) * s
        c0, c1 = g.mean(), (g * xh).mean()
        want = s * (g - c0 - xh * c1)
        # xh: three roundings, of differences no larger than |x| + |mean|
        e_xh = 3 * U * (v[r].abs() + abs(float(mean[r]))) * s
        e0, e1 = K * U * g.abs().mean(), (K + 2) * U * (g * xh).abs().mean() + (g.abs() * e_xh).mean()
        bound = s * (e0 + xh.abs() * e1 + e_xh * c1.abs() + 4 * U * (g.abs() + c0.abs() + (xh * c1).abs())) + 2 * U * want.abs()
        assert bool(((dx[r].double() - want).abs() <= bound).all())
        sums[0] += g * xh
        sums[1] += g
    assert bool(((db.double() - sums[1]).abs() <= (M + 40) * U * dy.double().abs().sum(0)).all())
    size = (dy.double().abs() * (v.abs() + mean.double().abs()[:, None]) * rstd.double()[:, None]).sum(0)
    assert bool(((dg.double() - sums[0]).abs() <= (M + 44) * U * size).all())


@pytest.mark.parametrize("C", [40, 1000, 4096, 12000, 40000])
@pytest.mark.parametrize("dtype", [F, B])
def test_parameters_and_statistics_on_any_boundary(C, dtype):
    """The bits of a call do not depend on where gamma, beta and the vectors lie, as far as their boundaries choose the same kernel; all of them are right."""
    M = 300
    x, dy = _randn(1, M, C).to(dtype), _randn(2, M, C).to(dtype)
    ga, be = 1 + 0.3 * _randn(3, C), 0.3 * _randn(4, C)

    def off(t, k):
        out = torch.empty(t.numel() + 4, device="cuda")[k:k + t.numel()]
        return out.copy_(t)

    v = x.double()
    d = v - v.mean(1, keepdim=True)
    want_rstd = 1.0 / (d.square().mean(1) + EPS).sqrt()
    xh = d * want_rstd[:, None]
    want = xh * ga.double() + be.double()
    g = dy.double() * ga.double()
    want_dx = want_rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    for k in range(4):
        y = torch.empty(M, C, dtype=dtype, device="cuda")
        mean, rstd = off(torch.zeros(M, device="cuda"), k), off(torch.zeros(M, device="cuda"), (k + 1) % 4)
        twn.layer_norm_fwd(x, C, M, C, off(ga, k), off(be, (k + 2) % 4), EPS, y, C, mean, rstd)
        dx, dg, db = torch.empty(M, C, dtype=dtype, device="cuda"), off(torch.zeros(C, device="cuda"), k), off(torch.zeros(C, device="cuda"), (k + 3) % 4)
        twn.layer_norm_bwd(dy, C, x, C, M, C, off(ga, k), mean, rstd, dx, C, dg, db, workspace(twn.layer_norm_bwd_workspace_bytes(M, C)))
        # sums of some hundred roundings of terms of size 1, of elements below 6
        bar = 100 * 6 * 6 * U
        assert bool(((y.double() - want).abs() <= bar + HALF[dtype] * want.abs()).all())
        assert bool(((dx.double() - want_dx).abs() <= bar * float(want_rstd.max()) + HALF[dtype] * want_dx.abs()).all())
        assert bool(((dg.double() - (dy.double() * xh).sum(0)).abs() <= M * 36 * 2 * U).all())
        assert bool(((db.double() - dy.double().sum(0)).abs() <= M * 6 * 2 * U).all())


def test_more_rows_than_32_bits_count():
    """Rows of two: x = m + d and m - d give 1 and -1 (times d / sqrt(d^2 + eps)); whole numbers, so that sums over the rows are exact."""
    M, C = (1 << 31) + 1003, 2
    x = torch.empty(M, C, dtype=B, device="cuda")
    x[:, 0], x[:, 1] = 3.0, 1.0
    x[-5:, 0] = 5.0
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    twn.layer_norm_fwd(x, C, M, C, None, None, 0.0, y, C, mean, rstd)
    assert bool((y[:, 0] == 1.0).all()) and bool((y[:, 1] == -1.0).all())
    assert bool((mean[:-5] == 2.0).all()) and bool((mean[-5:] == 3.0).all()) and bool((rstd[:-5] == 1.0).all()) and bool((rstd[-5:] == 0.5).all())
    # a gradient in few rows: dgamma = sum dy xh, dbeta = sum dy; dx = rstd (dy - (dy0 + dy1) / 2 - xh (dy0 - dy1) / 2) = 0 for two channels
    dy = torch.zeros_like(x)
    rows = [0, 1, 12345, (1 << 31) - 1, 1 << 31, (1 << 31) + 1, M - 1]
    for i, r in enumerate(rows):
        dy[r, 0], dy[r, 1] = float(i + 1), 2.0
    dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    del y
    dx = torch.full_like(x, 7.0)
    ws = workspace(twn.layer_norm_bwd_workspace_bytes(M, C))
    twn.layer_norm_bwd(dy, C, x, C, M, C, None, mean, rstd, dx, C, dg, db, ws)
    assert bool((dx == 0).all())
    assert dg.tolist() == [28.0, -14.0] and db.tolist() == [28.0, 14.0]
