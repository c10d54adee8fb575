"""twn_orthogonalize_batch and twn_muon_update_batch refuse what they cannot serve on the host, before any CUDA call."""
import ctypes as C

import pytest

from paper_1605_04711_b200 import build, twn

INVALID, MISALIGNED, WORKSPACE, TOO_LARGE = -1, -2, -3, -9
FAKE = 1 << 20                   # never dereferenced: a host check comes first


@pytest.fixture(scope="module")
def lib():
    lib = C.CDLL(build.build())
    lib.twn_orthogonalize_workspace_bytes.restype = lib.twn_muon_workspace_bytes.restype = C.c_size_t
    return lib


def orthogonalize(lib, rows=8, cols=8, G=FAKE, O=FAKE, gt=0, ot=0, count=1, steps=5, eps=1e-7, ws=FAKE, size=1 << 40, status=0, items=True):
    it = (twn._OrthogonalizeItem * max(1, min(count, 40)))(*[twn._OrthogonalizeItem(G, O, rows, cols, gt, ot)] * max(0, min(count, 40)))
    return lib.twn_orthogonalize_batch(it if items else None, count, steps, C.c_double(eps), C.c_void_p(ws), C.c_size_t(size), C.c_void_p(status), None)


def muon(lib, rows=8, cols=8, W=FAKE, dW=FAKE, V=FAKE, stats=FAKE, count=1, lr=0.1, mu=0.9, wd=0.0, look=1, steps=5, eps=1e-7, factor=0.7, ws=FAKE,
         size=1 << 40):
    it = (twn._MuonItem * max(1, min(count, 40)))(*[twn._MuonItem(W, dW, V, rows, cols, stats)] * max(0, min(count, 40)))
    f = C.c_float
    return lib.twn_muon_update_batch(it, count, f(lr), f(mu), f(wd), look, steps, C.c_double(eps), C.c_double(factor), C.c_void_p(ws), C.c_size_t(size),
                                     None, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("args,code", [
    ({"count": -1}, INVALID), ({"count": 33}, INVALID), ({"items": False}, INVALID), ({"steps": 0}, INVALID), ({"steps": 33}, INVALID),
    ({"eps": 0.0}, INVALID), ({"eps": -1.0}, INVALID), ({"eps": NAN}, INVALID), ({"eps": INF}, INVALID), ({"eps": 1e-31}, INVALID),
    ({"rows": -1}, INVALID), ({"cols": -1}, INVALID), ({"gt": 2}, INVALID), ({"ot": -1}, INVALID), ({"G": 0}, INVALID), ({"O": 0}, INVALID),
    ({"ws": 0}, INVALID), ({"rows": 32769, "cols": 32769}, TOO_LARGE), ({"rows": (1 << 24) + 1}, TOO_LARGE),
    ({"rows": 32768, "cols": 1 << 24, "count": 32, "size": 1 << 63}, TOO_LARGE),
    ({"G": FAKE + 2}, MISALIGNED), ({"O": FAKE + 2}, MISALIGNED), ({"G": FAKE + 1, "gt": 1}, MISALIGNED), ({"ws": FAKE + 16}, MISALIGNED),
    ({"status": FAKE + 2}, MISALIGNED), ({"size": 1024}, WORKSPACE), ({"count": 0}, 0), ({"count": 0, "items": False, "ws": 0}, 0),
    ({"rows": 0}, 0), ({"cols": 0, "G": 0, "O": 0}, 0)])
def test_orthogonalize(lib, args, code):
    assert orthogonalize(lib, **args) == code


@pytest.mark.parametrize("args,code", [
    ({"count": -1}, INVALID), ({"count": 33}, INVALID), ({"lr": NAN}, INVALID), ({"mu": NAN}, INVALID), ({"wd": NAN}, INVALID), ({"look": 2}, INVALID),
    ({"steps": 0}, INVALID), ({"eps": 0.0}, INVALID), ({"factor": -1.0}, INVALID), ({"factor": NAN}, INVALID), ({"W": 0}, INVALID), ({"dW": 0}, INVALID),
    ({"V": 0}, INVALID), ({"W": FAKE + 4}, MISALIGNED), ({"dW": FAKE + 4}, MISALIGNED), ({"V": FAKE + 8}, MISALIGNED), ({"stats": FAKE + 4}, MISALIGNED),
    ({"ws": 0}, INVALID), ({"ws": FAKE + 8}, MISALIGNED), ({"size": 4096}, WORKSPACE), ({"rows": 40000, "cols": 40000}, TOO_LARGE), ({"count": 0}, 0)])
def test_muon(lib, args, code):
    assert muon(lib, **args) == code


@pytest.mark.parametrize("big", [0, 100])
def test_matrices_that_overlap_are_refused(lib, big):
    """An output over another matrix's input or output, over a part of its own input, or over it in another type."""
    def call(*items):
        its = (twn._OrthogonalizeItem * len(items))(*[twn._OrthogonalizeItem(g, o, 8 + 50 * big, 8 + big, gt, ot) for g, o, gt, ot in items])
        size = lib.twn_orthogonalize_workspace_bytes(its, len(items))
        return lib.twn_orthogonalize_batch(its, len(items), 5, C.c_double(1e-7), C.c_void_p(FAKE), C.c_size_t(size), None, None)

    n = (8 + 50 * big) * (8 + big) * 4
    x = [(1 << 30) + i * n for i in range(4)]
    refused = [[(x[0], x[1], 0, 0), (x[1], x[2], 0, 0)], [(x[1], x[2], 0, 0), (x[0], x[1], 0, 0)], [(x[0], x[2], 0, 0), (x[1], x[2], 0, 0)],
               [(x[0], x[0], 0, 0)] * 2, [(x[0], x[0] + 4, 0, 0)], [(x[0] + n - 4, x[0], 0, 0)], [(x[0], x[0], 0, 1)], [(x[0], x[0], 1, 0)]]
    for items in refused:
        assert call(*items) == INVALID
    # one input for two outputs, in place, side by side: what stops these is that there is no device
    for items in [[(x[0], x[1], 0, 0), (x[0], x[2], 0, 0)], [(x[0], x[0], 0, 0), (x[1], x[1], 1, 1)], [(x[1], x[0], 0, 0), (x[1], x[2], 0, 0)]]:
        assert _no_device() and call(*items) not in (INVALID, MISALIGNED, WORKSPACE, TOO_LARGE)


def _no_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")
    return True


def test_muon_matrices_that_overlap_are_refused(lib):
    n = 64 * 64 * 4
    x = [(1 << 30) + i * n for i in range(8)]

    def call(*items):
        its = (twn._MuonItem * len(items))(*[twn._MuonItem(w, d, v, 64, 64, 0) for w, d, v in items])
        size = lib.twn_muon_workspace_bytes(its, len(items))
        f = C.c_float
        return lib.twn_muon_update_batch(its, len(items), f(0.1), f(0.9), f(0.0), 1, 5, C.c_double(1e-7), C.c_double(0.7), C.c_void_p(FAKE),
                                         C.c_size_t(size), None, None)

    for items in [[(x[0], x[0], x[1])], [(x[0], x[1], x[0])], [(x[0], x[1], x[1])], [(x[0], x[1], x[2])] * 2, [(x[0], x[1], x[2]), (x[3], x[4], x[2])],
                  [(x[0], x[1], x[2]), (x[1], x[4], x[5])], [(x[0], x[1], x[2]), (x[3], x[0] + n - 16, x[5])]]:
        assert call(*items) == INVALID
    for items in [[(x[0], x[1], x[2]), (x[3], x[1], x[4])], [(x[0], x[1], x[2]), (x[3], x[4], x[5])]]:
        assert _no_device() and call(*items) not in (INVALID, MISALIGNED, WORKSPACE, TOO_LARGE)



def test_workspace():
    one, two = twn.orthogonalize_workspace_bytes([(64, 576)]), twn.orthogonalize_workspace_bytes([(64, 576), (576, 64)])
    assert 0 < one < two and one % 256 == 0
    assert twn.muon_workspace_bytes([(64, 576)]) >= one + 64 * 576 * 4
    assert twn.orthogonalize_workspace_bytes([(32769, 32769)]) == 0 and twn.orthogonalize_workspace_bytes([(1, 1)] * 33) == 0
    assert twn.orthogonalize_workspace_bytes([(-1, 1)]) == 0 and twn.orthogonalize_workspace_bytes([]) > 0


def test_binding_refuses_tensors_that_are_not_on_the_device():
    import torch
    x = torch.zeros(4, 4)
    with pytest.raises(AssertionError):
        twn.orthogonalize_batch([(x, 4, 4, x)], 5, 1e-7, x)
