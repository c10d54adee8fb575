"""The sums over the rows of a layer norm's backward pass, to the last row.

dY, X and the statistics are small whole numbers (mean 1, 1 / deviation 1 or 2), so every product and every partial sum is a whole
number below 2^24, which fp32 holds exactly whatever the order: dgamma and dbeta have to be equal to the sums of 64 bits.  A row
that is lost or counted twice changes them by whole numbers.
"""
import pytest
import torch

from paper_1605_04711_b200 import twn
from _gpu_util import workspace

pytestmark = pytest.mark.gpu

F, B = torch.float32, torch.bfloat16


@pytest.mark.parametrize("M,C", [(1, 16), (2, 7), (147, 33), (148, 64), (149, 64), (5000, 24), (5000, 212), (9000, 1001), (20011, 64), (200704, 64), (4099, 4096), (4100, 260), (2999, 1001), (60000, 100),
                                 (149, 8192), (1031, 8200), (700, 16384), (300, 12004), (297, 9001), (150, 20000), (41, 32768), (600, 17000), (3, 50001)])
@pytest.mark.parametrize("dt,xt", [(F, F), (B, B), (F, B), (B, F)])
def test_no_row_is_lost_or_counted_twice(M, C, dt, xt):
    g = torch.Generator(device="cuda").manual_seed(M + C)
    # |dY| <= 3, |X - mean| <= 4, 1 / deviation <= 2: the sums stay below 24 M < 2^24 for the most rows here, and each row counts
    dy = torch.randint(-3, 4, (M, C), generator=g, device="cuda")
    x = torch.randint(-3, 6, (M, C), generator=g, device="cuda")
    mean, rstd = torch.ones(M, device="cuda"), torch.randint(1, 3, (M,), generator=g, device="cuda").float()
    dg, db = (torch.full((C,), 9.0, device="cuda") for _ in range(2))
    ws = workspace(twn.layer_norm_bwd_workspace_bytes(M, C))
    ws.fill_(255)
    dX = torch.empty(M, C, dtype=dt, device="cuda")
    for out in (dX, None):
        twn.layer_norm_bwd(dy.to(dt), C, x.to(xt), C, M, C, None, mean, rstd, out, C, dg, db, ws)
        assert torch.equal(dg.double(), (dy.double() * (x.double() - 1) * rstd.double()[:, None]).sum(0))
        assert torch.equal(db.double(), dy.double().sum(0))
