"""Row strides of the operators on scores whose products leave 64 bits, without a
GPU: they are refused before anything is enqueued.  Of one row, or shared by all
rows, a stride means nothing or is 0."""
import pytest

from tests.test_policy import ENOSPACE, ESHAPE, _balance, _constrain, _constraints, lib  # noqa: F401  (a fixture)

FAR = 1 << 62   # 4 rows of it are 0 modulo 2^64 elements


@pytest.mark.parametrize("kw", [
    dict(xs=FAR), dict(ps=FAR), dict(out=1 << 25, os=FAR), dict(xs=(1 << 56) + 1), dict(dtype=1, xs=(1 << 63) - 1),
    dict(c=_constraints(allow=1 << 29, allow_stride=FAR)), dict(c=_constraints(bias=1 << 29, bias_stride=FAR)),
    dict(c=_constraints(history=1 << 29, n_history=9, history_stride=FAR)),
])
def test_constrain_refuses_strides_whose_products_leave_64_bits(lib, kw):   # noqa: F811
    assert _constrain(lib, **kw) == ESHAPE
    assert b"span" in lib.tag_last_error()


@pytest.mark.parametrize("kw", [dict(xs=FAR), dict(gs=FAR), dict(xs=(1 << 56) + 1), dict(gs=(1 << 63) - 1)])
def test_balance_refuses_strides_whose_products_leave_64_bits(lib, kw):   # noqa: F811
    assert _balance(lib, **kw) == ESHAPE
    assert b"span" in lib.tag_last_error()


def test_strides_that_mean_nothing(lib):   # noqa: F811
    """They pass: what is refused is the workspace."""
    free = dict(allow=1 << 29, bias=1 << 30, history=1 << 31, n_history=9)
    S = 70000
    big = dict(S=S, xs=FAR, ps=FAR, out=1 << 25, os=FAR)
    assert _constrain(lib, Q=1, c=_constraints(**free, allow_stride=FAR, bias_stride=FAR, history_stride=FAR), **big) == ENOSPACE
    big = dict(S=S, xs=1 << 30, ps=1 << 30, out=1 << 50, os=1 << 30, prior=1 << 54)
    assert _constrain(lib, Q=4, c=_constraints(**free), **big) == ENOSPACE
    unused = _constraints(allow_stride=FAR, bias_stride=FAR, history_stride=FAR)   # (of arrays that are not there)
    assert _constrain(lib, Q=4, c=unused, **big) == ENOSPACE
    assert _balance(lib, Q=1, xs=FAR, gs=FAR, nb=16) == ENOSPACE
