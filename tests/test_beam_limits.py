"""Row strides of a beam search's scores whose products leave 64 bits, without a GPU:
they are refused before anything is enqueued."""
import pytest

from tests.test_beam import ESHAPE, _select, lib  # noqa: F401  (a fixture)


@pytest.mark.parametrize("kw", [
    dict(xs=1 << 62),                                     # (5 rows of it are 0 modulo 2^64 bytes)
    dict(xs=(1 << 62) // 5 * 4, dtype=1), dict(xs=(1 << 63) - 1), dict(n=1, V=2, xs=(1 << 57) + 1),
    dict(n=1 << 21, V=256, W=256, xs=(1 << 29) + 1, x=1 << 50),
])
def test_strides_whose_products_leave_64_bits(lib, kw):   # noqa: F811
    assert _select(lib, **kw) == ESHAPE
    assert b"span" in lib.tag_last_error()
