"""Strides of matrices whose products leave 64 bits, without a GPU: they are refused
before anything is enqueued.  Of one row or one matrix a stride means nothing.  A
call that passes its checks ends at the workspace, which is too small."""
import ctypes as C

import pytest

from tests.test_optim_overlap import BASE, ENOSPACE, _muon, _ortho, abi  # noqa: F401  (a fixture)

ESHAPE = -4
FAR = 1 << 62


# (offset, row stride, matrix stride); 4 matrices, or 9 rows, of FAR are little modulo 2^64
@pytest.mark.parametrize("shape,far,near", [
    ((5, 8, 6), (0, 6, FAR), (1 << 20, 6, 48)), ((1, 9, 6), (0, FAR, 0), (1 << 20, 6, 0)),
    ((5, 8, 6), (0, FAR, 48), (1 << 20, 6, 48)), ((5, 8, 6), (0, 6, (1 << 63) - 1), (1 << 20, 6, 48)),
    ((4, 8, 6), (0, 6, (1 << 56) + 1), (1 << 20, 6, 48)), ((1, 8, 6), (0, (1 << 55) + 1, 0), (1 << 20, 6, 0)),
])
def test_strides_whose_products_leave_64_bits(abi, shape, far, near):   # noqa: F811
    third = (1 << 24,) + near[1:]
    for plain in (0, 1):
        for arrays in ((far, near, third), (near, far, third), (near, third, far)):
            assert _muon(abi, shape, *arrays, plain=plain) == ESHAPE
            assert b"span" in abi.load().tag_last_error()
    for dtype in (0, 1):
        for x, y in ((far, near), (near, far), (far, far)):
            assert _ortho(abi, shape, x, y, dtype) == ESHAPE


def test_strides_that_mean_nothing(abi):   # noqa: F811
    one = ((0, FAR, FAR), (1 << 20, FAR, FAR), (1 << 24, FAR, FAR))
    assert _muon(abi, (1, 1, 60), *one) == ENOSPACE and _ortho(abi, (1, 1, 60), *one[:2]) == ENOSPACE
    rows = ((0, 1 << 50, FAR), (1 << 20, 90, FAR), (1 << 24, 90, FAR))
    assert _muon(abi, (1, 70, 90), *rows) == ENOSPACE and _ortho(abi, (1, 70, 90), *rows[:2]) == ENOSPACE
