"""The workspaces of group norm: as much as a call has sums for, and enough for any smaller batch."""
import ctypes as C

import pytest

from paper_1605_04711_b200 import build

i64 = C.c_int64


@pytest.fixture(scope="module")
def sizes():
    lib = C.CDLL(build.build())
    fns = lib.twn_group_norm_fwd_workspace_bytes, lib.twn_group_norm_bwd_workspace_bytes
    for f in fns:
        f.restype = C.c_size_t
    return [lambda B, HW, Cc, G, f=f: f(i64(B), i64(HW), i64(Cc), G) for f in fns]


@pytest.mark.parametrize("B,HW,Cc,G", [(4096, 49, 512, 32), (4096, 1, 512, 32), (20000, 4, 64, 8), (1000, 196, 256, 32)])
def test_of_small_images(sizes, B, HW, Cc, G):
    """A block has an image, whole or some channels of it, or at most half of one: two sums of a channel and a block."""
    assert B * 2 * Cc * 4 <= sizes[1](B, HW, Cc, G) <= 2 * B * 2 * Cc * 4


SHAPES = [(49, 512, 32), (1, 512, 32), (3136, 256, 32), (12544, 64, 32), (1501, 200, 8), (65536, 24, 8), (131072, 512, 1), (1000, 51, 1), (20000, 50, 2), (784, 990, 33), (5, 7, 7),
          (300, 1030, 2), (50, 16384, 1), (40000, 48, 1)]


@pytest.mark.parametrize("HW,Cc,G", SHAPES, ids=str)
def test_fewer_images_need_no_more(sizes, HW, Cc, G):
    for size in sizes:
        last = 0
        for B in list(range(1, 160)) + [200, 295, 296, 297, 400, 591, 592, 593, 700, 1183, 1184, 1185, 3000]:
            now = size(B, HW, Cc, G)
            assert now >= last and now % 256 == 0, B
            last = now
