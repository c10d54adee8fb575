"""twn_layer_norm_fwd and twn_layer_norm_bwd refuse what they cannot serve on the host, before any CUDA call."""
import ctypes as C

import pytest

from paper_1605_04711_b200 import build

INVALID, MISALIGNED, WORKSPACE, TOO_LARGE = -1, -2, -3, -9
F32, BF16 = 0, 1
FAKE, ODD = 1 << 20, (1 << 20) + 2          # never dereferenced: a host check comes first


@pytest.fixture(scope="module")
def lib():
    lib = C.CDLL(build.build())
    lib.twn_layer_norm_bwd_workspace_bytes.restype = C.c_size_t
    return lib


def _ptr(p):
    return C.c_void_p(p)


def fwd(lib, X=FAKE, xt=F32, ldx=64, M=4, Cc=64, gamma=FAKE, beta=FAKE, eps=1e-5, Y=FAKE, yt=F32, ldy=64, mean=0, rstd=0):
    i = C.c_int64
    return lib.twn_layer_norm_fwd(_ptr(X), xt, i(ldx), i(M), i(Cc), _ptr(gamma), _ptr(beta), C.c_double(eps), _ptr(Y), yt, i(ldy),
                                  _ptr(mean), _ptr(rstd), None)


def bwd(lib, dY=FAKE, dt=F32, lddy=64, X=FAKE, xt=F32, ldx=64, M=4, Cc=64, gamma=FAKE, mean=FAKE, rstd=FAKE, dX=FAKE, ot=F32, lddx=64, residual=0,
        dgamma=FAKE, dbeta=FAKE, ws=FAKE, bytes_=None):
    i = C.c_int64
    if bytes_ is None:
        bytes_ = lib.twn_layer_norm_bwd_workspace_bytes(i(4), i(64))
    return lib.twn_layer_norm_bwd(_ptr(dY), dt, i(lddy), _ptr(X), xt, i(ldx), i(M), i(Cc), _ptr(gamma), _ptr(mean), _ptr(rstd), _ptr(dX), ot,
                                  i(lddx), _ptr(residual), _ptr(dgamma), _ptr(dbeta), _ptr(ws), C.c_size_t(bytes_), None)


@pytest.mark.parametrize("args,code", [
    ({"M": -1}, INVALID), ({"Cc": 0}, INVALID), ({"Cc": -3}, INVALID), ({"Cc": 65}, INVALID), ({"ldy": 63}, INVALID),
    ({"X": 0}, INVALID), ({"Y": 0}, INVALID), ({"xt": 2}, INVALID), ({"yt": -1}, INVALID), ({"eps": -1e-9}, INVALID),
    ({"eps": float("nan")}, INVALID), ({"eps": float("inf")}, INVALID), ({"Cc": (1 << 31) + 1, "ldx": 1 << 32, "ldy": 1 << 32}, INVALID),
    ({"X": ODD}, MISALIGNED), ({"Y": ODD}, MISALIGNED), ({"X": FAKE + 1, "xt": BF16}, MISALIGNED), ({"gamma": ODD}, MISALIGNED),
    ({"mean": ODD}, MISALIGNED), ({"ldx": 1 << 60}, TOO_LARGE), ({"M": 1 << 57}, TOO_LARGE), ({"M": 0}, 0), ({"M": 0, "X": 0, "Y": 0}, 0)])
def test_forward(lib, args, code):
    assert fwd(lib, **args) == code


@pytest.mark.parametrize("args,code", [
    ({"M": -1}, INVALID), ({"Cc": 0}, INVALID), ({"lddy": 63}, INVALID), ({"ldx": 63}, INVALID), ({"lddx": 63}, INVALID), ({"dY": 0}, INVALID),
    ({"X": 0}, INVALID), ({"mean": 0}, INVALID), ({"rstd": 0}, INVALID), ({"dt": 2}, INVALID), ({"xt": 3}, INVALID), ({"ot": 5}, INVALID),
    ({"dY": ODD}, MISALIGNED), ({"dX": ODD}, MISALIGNED), ({"dgamma": ODD}, MISALIGNED), ({"ws": 0}, WORKSPACE), ({"bytes_": 16}, WORKSPACE),
    ({"ws": FAKE + 16}, MISALIGNED), ({"lddx": 1 << 60}, TOO_LARGE), ({"dX": 0, "dgamma": 0, "dbeta": 0, "ws": 0}, 0),
    ({"M": 0, "dgamma": 0, "dbeta": 0}, 0), ({"residual": ODD}, MISALIGNED), ({"residual": FAKE, "dX": 0}, INVALID)])
def test_backward(lib, args, code):
    assert bwd(lib, **args) == code


def test_workspace(lib):
    size = lambda M, Cc: lib.twn_layer_norm_bwd_workspace_bytes(C.c_int64(M), C.c_int64(Cc))  # noqa: E731
    assert size(1, 1) > 0 and size(1, 1) % 256 == 0 and size(0, 64) > 0
    assert size(-1, 4) == 0 and size(4, 0) == 0
    assert size(100, 4096) >= size(100, 64) and size(10000, 64) >= size(1, 64)


def test_binding_refuses_tensors_that_are_not_on_the_device():
    import torch
    from paper_1605_04711_b200 import twn
    x = torch.zeros(4, 64)
    with pytest.raises(AssertionError):
        twn.layer_norm_fwd(x, 64, 4, 64, None, None, 1e-5, x, 64)
