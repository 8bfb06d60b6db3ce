"""The largest calls of the operators on scores: a launch of 2^32 threads and more,
its last block included, is refused before anything is enqueued."""
import ctypes as C

import pytest

from tests.test_policy import ESHAPE, _constrain, lib  # noqa: F401  (a fixture)


@pytest.mark.parametrize("Q,S", [
    (2 ** 28 - 1, 1), (2 ** 28 - 15, 256), (2 ** 28 - 8, 60),   # sixteen rows to a block of 256 threads
    (2 ** 26 - 1, 257), (2 ** 26 - 3, 1024),                    # four
    (2 ** 24, 1025), (2 ** 23, 4097), (2 ** 22, 8193),          # one
    (2 ** 20, 16 * 4096), (2 ** 19, 31 * 4096 + 1),             # parts of 4,096 columns
])
def test_constrain_refuses_launches_of_2_32_threads(lib, Q, S):   # noqa: F811
    kw = dict(Q=Q, S=S, xs=S, ps=S, x=1 << 48, prior=None, nb=1 << 62)
    assert _constrain(lib, **kw) == ESHAPE
    b = C.c_size_t(0)
    assert lib.tag_constrain_workspace(Q, S, C.byref(b)) == 0
