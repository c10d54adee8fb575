"""1 / deviation of group norm, to its last digits."""
import pytest
import torch

from test_gpu_group_norm import U, fwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C,G", [(64, 32), (24, 24), (32, 16)])
def test_of_an_exact_variance(C, G):
    """Values of +-d, with d a power of two times 1 to 2 of eleven bits: sums and squares are exact, whichever way they are split, and so is the mean, 0.  What is left are a rounding of the
    variance plus eps and that of the root's reciprocal: 1/deviation is off by half a step for the latter and a quarter (half of a half) for the former; 1.6 u allows for eps in fp32."""
    B, HW = 64, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    d = torch.randint(1024, 2048, (B, 1, G, 1), device="cuda", generator=g).float() / 1024 * 2.0 ** torch.randint(-3, 4, (B, 1, G, 1), device="cuda", generator=g)
    sign = torch.ones(HW, device="cuda")
    sign[1::2] = -1.0
    X = (d * sign.view(1, HW, 1, 1)).expand(B, HW, G, C // G).reshape(-1).contiguous()
    mean, rstd, Y = torch.empty(B * G, device="cuda"), torch.empty(B * G, device="cuda"), torch.empty_like(X)
    eps = 2.0 ** -16
    fwd(X, C, B, HW, C, G, None, None, "none", Y, C, mean, rstd, eps=eps)
    assert bool((mean == 0).all())
    want = (d.double().view(-1) ** 2 + eps).rsqrt()
    off = (rstd.double() / want - 1.0).abs() / U
    assert float(off.max()) <= 1.6, float(off.max())
