"""The factor that clips gradients whose norm is above all numbers of fp32."""
import math

import pytest
import torch

from paper_1605_04711_b200 import twn

pytestmark = pytest.mark.gpu


def test_finite_gradients_with_a_norm_above_fp32():
    """The factor comes from the norm in 64 bits; the norm that is written is infinite, as fp32 has it."""
    n = 100_000
    for value, limit in ((3e38, 1e38), (3e38, 1.0), (2e37, 1e37)):
        g = torch.full((n,), value, device="cuda")
        norm, scale = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
        ws = torch.empty(twn.grad_norm_workspace_bytes([n]), dtype=torch.uint8, device="cuda")
        twn.grad_norm_batch([g], limit, norm, scale, ws)
        want = limit / (math.sqrt(n) * float(g[0].double()))
        assert float(norm) == float("inf")
        # one rounding of fp32, of a number that may lie below 2^-126
        assert abs(float(scale) - want) <= 2.0 ** -24 * want * 1.001 + 2.0 ** -150
        twn.grad_norm_batch([g, torch.tensor([float("inf")], device="cuda")], limit, norm, scale, torch.empty(twn.grad_norm_workspace_bytes([n, 1]), dtype=torch.uint8, device="cuda"))
        assert float(norm) == float("inf") and float(scale) == 0.0
