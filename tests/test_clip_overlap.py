"""Clipping refuses outputs that share memory with one another or with another gradient (before any GPU work: this runs
without one), and takes all that do not."""
import ctypes as C

import pytest

from paper_2402_14212_b200 import binding as mwb

INVALID, WORKSPACE = 1, 3


def call(src, dst, sizes, kinds=None, most=1.0):
    """With a scratch that is refused, so that nothing is launched: what the checks before it say."""
    n, L = len(src), mwb.lib()
    kinds = kinds or [1] * n
    ptr = lambda v: (C.c_void_p * n)(*v)
    return L.mw_clip_gradients(n, ptr(src), None if dst is None else ptr(dst), (C.c_int64 * n)(*sizes), (C.c_int32 * n)(*kinds), most, 256, None, 0,
                               None)


INF = float("inf")


@pytest.mark.parametrize("src,dst,sizes", [
    ([4096, 4096], [4096, 4096], [10, 10]),                     # one tensor twice
    ([4096, 8192], [12288, 12288], [10, 10]),                   # one output twice
    ([4096, 8192], [12288, 12288 + 36], [10, 10]),              # ... or nearly
    ([8192, 4096, 4132], [8192, 4096, 4132], [5, 10, 3]),       # a window of another
    ([4096, 8192], [8192, 4096], [10, 10]),                     # each other's place
    ([4096, 8192], [12288, 4100], [10, 10]),                    # another's input
    ([4096], [4100], [10]),                                     # its own, shifted
    ([4096, 8192], [8192 - 36, 16384], [10, 10]),
])
def test_shared_memory_is_refused(src, dst, sizes):
    assert call(src, dst, sizes) == INVALID
    if src != dst:
        assert call(src, dst, sizes, most=INF) == INVALID


def test_what_is_apart_passes():
    many = [4096 + 40 * i for i in range(600)]
    for src, dst, sizes in (([4096, 4136], [4096, 4136], [10, 10]), (many, many, [10] * 600), (many[::-1], many[::-1], [10] * 600),
                            (many, [m + 600 * 40 for m in many[::-1]], [10] * 600), ([4096, 4096], [8192, 12288], [10, 10]),
                            ([4096, 4100, 4096], [4096, 4100, 0], [1, 5, 0]), ([4096, 4096], [4096, 4116], [10, 0])):
        assert call(src, dst, sizes) == WORKSPACE
    # bf16 tensors are half as long
    assert call([4096, 4116], [4096, 4116], [10, 10], [2, 1]) == WORKSPACE
    assert call([4096, 4116], [4096, 4116], [10, 10], [1, 2]) == INVALID
    # the norm alone writes nothing
    assert call([4096, 4096], None, [10, 10], most=INF) == call([4096, 4096], [4096, 4096], [10, 10], most=INF) == WORKSPACE
