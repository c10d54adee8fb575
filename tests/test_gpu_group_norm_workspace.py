"""A workspace of group norm for a batch serves smaller ones, and nothing behind it is written."""
import pytest
import torch

from paper_1605_04711_b200 import twn
from test_gpu_group_norm import BF16, EPS, F32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,HW,C,G", [(64, 49, 512, 32), (40, 784, 64, 32), (9, 1501, 200, 8), (7, 40000, 48, 1), (34, 22000, 14, 7), (300, 4, 40, 5)], ids=str)
def test_smaller_batches(B, HW, C, G, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    X, dY = (torch.empty(B * HW * C, dtype=dtype, device="cuda").normal_(generator=g) for _ in range(2))
    sizes = twn.group_norm_fwd_workspace_bytes(B, HW, C, G), twn.group_norm_bwd_workspace_bytes(B, HW, C, G)

    def run(b, bytes_):
        ws = [torch.full((n + 4096,), 255, dtype=torch.uint8, device="cuda") for n in bytes_]
        n = b * HW * C
        x, dy, Y, dX = X[:n], dY[:n], torch.empty_like(X[:n]), torch.empty_like(X[:n])
        mean, rstd, dgamma, dbeta = (torch.empty(k, device="cuda") for k in (b * G, b * G, C, C))
        twn.group_norm_fwd(x, C, b, HW, C, G, None, None, EPS, twn.ACT_SILU, Y, C, mean, rstd, ws[0][:bytes_[0]])
        twn.group_norm_bwd(dy, C, x, C, b, HW, C, G, None, None, mean, rstd, twn.ACT_SILU, dX, C, dgamma, dbeta, ws[1][:bytes_[1]])
        assert all(bool((w[k:] == 255).all()) for w, k in zip(ws, bytes_))
        return Y, dX, mean, rstd, dgamma, dbeta

    for b in sorted({1, 2, B // 3, B - 1, B}):
        own = twn.group_norm_fwd_workspace_bytes(b, HW, C, G), twn.group_norm_bwd_workspace_bytes(b, HW, C, G)
        assert own[0] <= sizes[0] and own[1] <= sizes[1]
        for a, c in zip(run(b, sizes), run(b, own)):
            assert bool(a.isfinite().all()) and torch.equal(a, c)
