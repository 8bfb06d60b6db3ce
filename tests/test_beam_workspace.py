"""The workspace of a level of beam search, without a GPU: searches that fit one block
need none, rows in parts are refused without the whole of it."""
import ctypes as C

import pytest

from tests.test_beam import EINVAL, ENOSPACE, _select, lib  # noqa: F401  (a fixture)


def _need(lib, n, V, W, S):   # noqa: F811
    b = C.c_size_t(7)
    assert lib.tag_beam_workspace(n, V, W, S, C.byref(b)) == 0
    return b.value


@pytest.mark.parametrize("n,V,W,S", [(1, 1, 1, 16384), (2, 4, 4, 4096), (5, 64, 64, 256), (3, 256, 1, 60)])
def test_searches_of_one_block_need_none(lib, n, V, W, S):   # noqa: F811
    assert _need(lib, n, V, W, S) == 0


@pytest.mark.parametrize("n,V,W,S", [(1, 64, 64, 4097), (2, 1, 4, 16385), (3, 65, 1, 300), (8, 8, 8, 262140)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_in_parts_need_all_of_it(lib, n, V, W, S, dtype):   # noqa: F811
    need = _need(lib, n, V, W, S)
    # a maximum and a sum of each part of 4,096 columns, and maxima of groups of 16 columns or more
    parts, groups = n * V * ((S + 4095) // 4096), n * V * ((S + 15) // 16)
    assert 12 * parts < need <= 12 * parts + 4 * groups + 3 * 256   # (each array aligned)
    call = dict(n=n, V=V, W=W, S=S, xs=S, dtype=dtype, x=1 << 40)
    for kw, status in ((dict(nb=need - 1), ENOSPACE), (dict(nb=0, ws=None), ENOSPACE), (dict(nb=need, ws=None), EINVAL),
                       (dict(nb=need, ws=(1 << 25) + 8), EINVAL)):
        assert _select(lib, **call, **kw) == status, kw
        assert lib.tag_last_error()
