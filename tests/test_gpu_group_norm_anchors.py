"""Mean and variance of groups with a few values far from all others, wherever those lie among a thread's pixels, of which there may be hundreds.

Bounds.  A difference from what it is taken from is off by half a step of itself, u, and so is every addition of a thread; a run has at most 64 of those one after the other, of random
sign.  With K = 40 u as elsewhere: the mean is off by K times the mean size of the values at most, 1/deviation by K of itself."""
import pytest
import torch

from test_gpu_group_norm import BF16, F32
from test_gpu_group_norm_outliers import _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16])
@pytest.mark.parametrize("shape", [(2, 500, 64, 8), (1, 2000, 32, 4), (1, 90000, 24, 3), (2, 300, 24, 8), (3, 129, 7, 7), (2, 333, 150, 50)], ids=str)
def test_the_first_pixel(shape, dtype):
    """The first value of every group, and the whole first pixel, at 6e4: vectors of eight, eight pixels a thread and more."""
    B, HW, C, G = shape
    g = torch.Generator(device="cuda").manual_seed(1)
    for whole in (False, True):
        X = torch.randn(B, HW, C, device="cuda", generator=g)
        X[:, 0, ::1 if whole else C // G] = 6e4
        X = X.to(dtype).view(-1)
        Y, mean, rstd = _run(X, B, HW, C, G)
        _check(X, mean, rstd, B, HW, C, G, range(B))


# many pixels a thread: single bf16 elements of a tile in shared memory (about 200 and 400 pixels), vectors of two and four, and images that are read twice in one or a few tiles
MANY = [(160, 1000, 51, 1, BF16), (40, 15000, 51, 1, BF16), (160, 1000, 102, 1, BF16), (160, 700, 51, 1, F32), (160, 1000, 204, 1, BF16), (160, 1000, 408, 1, BF16),
        (600, 40000, 48, 1, BF16), (300, 20000, 51, 1, BF16), (300, 20000, 50, 2, F32)]


@pytest.mark.parametrize("shape", MANY, ids=lambda s: str(s[:4]))
def test_one_channel(shape):
    """One value of the first pixel at 6e4, and one of the last; of an image, which another image beside it has not."""
    B, HW, C, G, dtype = shape
    g = torch.Generator(device="cuda").manual_seed(2)
    X = torch.empty(B, HW, C, dtype=dtype, device="cuda").normal_(generator=g)
    for i, b in enumerate((0, 1, 2, 3, B - 1)):
        X[b, 0 if i != 1 else HW - 1, i::C // G] = 0.0
        X[b, 0 if i != 1 else HW - 1, 7 * i % (C // G)] = 6e4 if i % 2 == 0 else -3e4
    X = X.view(-1)
    _, mean, rstd = _run(X, B, HW, C, G)
    _check(X, mean, rstd, B, HW, C, G, (0, 1, 2, 3, 4, B - 1))


@pytest.mark.parametrize("shape", MANY[:3] + MANY[-3:], ids=lambda s: str(s[:4]))
def test_the_first_rows(shape):
    """The first pixels of an image, as many as a thread's first run has, are all far from the others; so are the last."""
    B, HW, C, G, dtype = shape
    g = torch.Generator(device="cuda").manual_seed(3)
    X = torch.empty(B, HW, C, dtype=dtype, device="cuda").normal_(generator=g)
    for b, at in ((0, slice(0, 64)), (1, slice(0, 320)), (2, slice(HW - 5, HW)), (3, slice(0, HW // 2))):
        X[b, at] += 3e4
    X = X.view(-1)
    _, mean, rstd = _run(X, B, HW, C, G)
    _check(X, mean, rstd, B, HW, C, G, range(5))


def test_far_from_zero_with_many_pixels():
    """Values around 1e4 with a deviation of 1, in fp32: the differences keep their digits (the roundings of the values themselves are in X)."""
    for B, HW, C, G in ((160, 700, 51, 1), (300, 20000, 50, 2), (2, 500, 64, 8)):
        g = torch.Generator(device="cuda").manual_seed(4)
        X = torch.empty(B, HW, C, device="cuda").normal_(1e4, 1.0, generator=g).view(-1)
        _, mean, rstd = _run(X, B, HW, C, G)
        _check(X, mean, rstd, B, HW, C, G, (0, 1, B - 1))
