"""A workspace of the orthogonalised updates that lies over a matrix is refused on the host."""
import ctypes as C

import pytest

from paper_1605_04711_b200 import twn
from test_orthogonalize_checks import INVALID, lib  # noqa: F401

BASE, FAR = 1 << 30, 1 << 36         # never dereferenced
N = 64 * 64 * 4


@pytest.fixture(autouse=True)
def _addresses_are_made_up():
    """A call that is served goes on to the device: these run only where there is none."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")


@pytest.mark.parametrize("rows", [64, 640])
def test_orthogonalize(lib, rows):  # noqa: F811
    def call(G, O, ws):
        it = (twn._OrthogonalizeItem * 1)(twn._OrthogonalizeItem(G, O, rows, 640, 0, 0))
        size = lib.twn_orthogonalize_workspace_bytes(it, 1)
        return size, lib.twn_orthogonalize_batch(it, 1, 5, C.c_double(1e-7), C.c_void_p(ws), C.c_size_t(size), None, None)

    size, code = call(BASE, FAR, 2 * FAR)
    assert code not in (INVALID, 0)
    n = rows * 640 * 4
    for G, O, ws in [(BASE, FAR, BASE), (BASE, FAR, FAR), (BASE, FAR, BASE - size + 256), (BASE, BASE, BASE + n - 256), (BASE, FAR, FAR - 256)]:
        assert call(G, O, ws)[1] == INVALID
    for G, O, ws in [(BASE, FAR, BASE + n), (BASE, BASE, BASE + n), (FAR, FAR + n, FAR - (size + 255) // 256 * 256)]:
        assert call(G, O, ws)[1] not in (INVALID, 0)


@pytest.mark.parametrize("which", range(3))
def test_muon(lib, which):  # noqa: F811
    at = [BASE, BASE + N, BASE + 2 * N]
    it = (twn._MuonItem * 1)(twn._MuonItem(*at, 64, 64, 0))
    size = lib.twn_muon_workspace_bytes(it, 1)
    f = C.c_float

    def call(ws):
        return lib.twn_muon_update_batch(it, 1, f(0.1), f(0.9), f(0.0), 1, 5, C.c_double(1e-7), C.c_double(0.7), C.c_void_p(ws), C.c_size_t(size), None, None)

    assert call(at[which]) == INVALID
    assert call(FAR) not in (INVALID, 0)
