"""The gates of group norm's ReLU where z leaves the range of fp32."""
import pytest
import torch

from test_gpu_group_norm import bwd

pytestmark = pytest.mark.gpu


def test_gates_of_tiny_values():
    """z that no fp32 number is: the gate of a ReLU is that of the formula in 64 bits."""
    HW, C, G = 64, 32, 4
    sign = (torch.arange(HW * C, device="cuda") % 3 - 1).float().view(HW, C)
    for x, ga, be, r in ((1e-25, 1e-25, 0.0, 1.0), (1e-30, 3e-10, 0.0, 1e-8), (1e20, 1e-20, 1e-20, 1e-20), (1.0, 0.0, 1.0, 1.0), (1.0, 0.0, 0.0, 1.0)):
        X = (sign * x).view(-1)
        gamma, beta = torch.full((C,), ga, device="cuda"), torch.full((C,), be, device="cuda")
        mean, rstd = torch.zeros(G, device="cuda"), torch.full((G,), r, device="cuda")
        dX, dbeta = torch.empty_like(X), torch.empty(C, device="cuda")
        bwd(torch.ones_like(X), C, X, C, 1, HW, C, G, gamma, beta, mean, rstd, "relu", dX, C, None, dbeta)
        z = X.double().view(HW, C) * rstd[0].double() * gamma.double() + beta.double()
        assert torch.equal(dbeta.double(), (z > 0).double().sum(0)), (x, ga, be, r)
