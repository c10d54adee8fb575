"""A layer norm's wait for a row that does not come, run to its limit on purpose (one millisecond, on a barrier nobody arrives on).  The
kernels have no status word: what such a row has touched is no number, and no wait after it is a long one."""
import ctypes as C

import pytest
import torch

from paper_1605_04711_b200 import twn

pytestmark = pytest.mark.gpu


def test_a_row_that_does_not_come_spoils_the_sums_and_nothing_hangs():
    sums, waits = torch.zeros(64, 8, device="cuda"), torch.full((64, 2), -1, dtype=torch.int32, device="cuda")
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    stream = torch.cuda.current_stream()
    t0.record()
    assert twn.lib().twn_selftest_row_wait(C.c_void_p(sums.data_ptr()), C.c_void_p(waits.data_ptr()), C.c_ulonglong(1_000_000), C.c_void_p(stream.cuda_stream)) == 0
    t1.record()
    torch.cuda.synchronize()
    assert t0.elapsed_time(t1) < 500.0
    assert bool((waits == 0).all()) and bool(sums.isnan().all())
    # the device is as it was
    x, y = torch.randn(2000, 1024, device="cuda"), torch.empty(2000, 1024, device="cuda")
    twn.layer_norm_fwd(x, 1024, 2000, 1024, None, None, 1e-5, y, 1024)
    want = torch.nn.functional.layer_norm(x.double(), (1024,))
    # |y| is below 6 in two million normal numbers; sums of 1024 and a few operations round to 2^-24 each, 64 of them in a row at most
    assert float((y.double() - want).abs().max()) <= 64 * 6 * 2.0 ** -24
