"""The operators on scores without a GPU: what their C entry points refuse
(before anything is enqueued), and the 64-bit restatements that the GPU tests
compare with, checked against differences and closed forms."""
import ctypes as C

import numpy as np
import pytest

from tests import _policy as R


@pytest.fixture(scope="module")
def lib():
    import paper_2302_06126_amd as P
    return P._abi.load()


EINVAL, ESHAPE, ENOSPACE = -1, -4, -5


def _constraints(**kw):
    from paper_2302_06126_amd._abi import tag_constraints
    c = tag_constraints()
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _constrain(lib, Q=4, S=100, dtype=0, x=1 << 20, xs=100, c=None, out=None, os=100, prior=1 << 24, ps=100,
               argmax=1 << 26, best=1 << 27, ws=1 << 28, nb=0):
    c = _constraints() if c is None else c
    return lib.tag_constrain(Q, S, dtype, x, xs, C.byref(c) if c else None, out, os, prior, ps, argmax, best, ws, nb,
                             None)


@pytest.mark.parametrize("kw,status", [
    (dict(Q=-1), EINVAL), (dict(S=0), EINVAL), (dict(dtype=2), EINVAL), (dict(x=None), EINVAL),
    (dict(argmax=None), EINVAL), (dict(best=None), EINVAL), (dict(xs=99), EINVAL), (dict(ps=99), EINVAL),
    (dict(out=1 << 25, os=99), EINVAL), (dict(x=(1 << 20) + 2), EINVAL), (dict(prior=(1 << 24) + 2), EINVAL),
    # constrained: the scores themselves row by row, or elsewhere
    (dict(out=1 << 20, os=104), EINVAL), (dict(out=(1 << 20) + 400), EINVAL), (dict(prior=(1 << 20) + 1200), EINVAL),
    (dict(out=1 << 24), EINVAL),
    (dict(c=_constraints(n_history=-1)), EINVAL), (dict(c=_constraints(n_history=3)), EINVAL),
    (dict(c=_constraints(history=1 << 29, n_history=9, history_stride=8)), EINVAL),
    (dict(c=_constraints(allow=1 << 29, allow_stride=3)), EINVAL),
    (dict(c=_constraints(bias=1 << 29, bias_stride=99)), EINVAL),
    (dict(c=_constraints(bias=(1 << 29) + 1)), EINVAL),
    # rows in parts need a workspace
    (dict(S=70000, xs=70000, ps=70000), ENOSPACE),
    (dict(S=70000, xs=70000, ps=70000, nb=1 << 20, ws=None), EINVAL),
    (dict(S=70000, xs=70000, ps=70000, nb=1 << 20, ws=(1 << 28) + 4), EINVAL),
    (dict(c=_constraints(history=1 << 22, n_history=(1 << 30) + 1)), ESHAPE),
    (dict(c=_constraints(repetition=(1 << 22) + 2)), EINVAL), (dict(best=(1 << 27) + 1), EINVAL),
    # (launches of 2^32 threads and more)
    (dict(Q=1 << 28, S=2, xs=2, ps=2, x=1 << 40, prior=1 << 44), ESHAPE),
    (dict(Q=1 << 24, S=3000, xs=3000, ps=3000, x=1 << 40, prior=1 << 44), ESHAPE),
    (dict(Q=1 << 22, S=1 << 28, xs=1 << 28, ps=1 << 28, x=0x1000, prior=1 << 61, nb=1 << 40), ESHAPE),
])
def test_constrain_refuses(lib, kw, status):
    assert _constrain(lib, **kw) == status
    assert lib.tag_last_error()


def test_constrain_of_no_rows_is_nothing(lib):
    assert _constrain(lib, Q=0, x=None, argmax=None, best=None) == 0
    assert lib.tag_constrain(1, 4, 0, 4096, 4, None, None, 0, None, 0, 4096, 4096, None, 0, None) == EINVAL


def test_workspaces(lib):
    b = C.c_size_t(7)
    assert lib.tag_constrain_workspace(5, 8192, C.byref(b)) == 0 and b.value == 0
    assert lib.tag_constrain_workspace(5, 262140, C.byref(b)) == 0 and 0 < b.value <= 5 * 262140
    assert lib.tag_constrain_workspace(5, 0, C.byref(b)) == EINVAL
    assert lib.tag_constrain_workspace(5, 10, None) == EINVAL
    assert lib.tag_balance_workspace(5, 16384, C.byref(b)) == 0 and b.value > 0
    assert lib.tag_balance_workspace(5, 16385, C.byref(b)) == ESHAPE
    assert lib.tag_balance_workspace(-1, 16, C.byref(b)) == EINVAL


def _balance(lib, Q=4, S=100, dtype=0, x=1 << 20, xs=100, mask=1 << 21, M=8, use=None, coef=0.5, grad=1 << 22, gs=100,
             acc=0, loss=1 << 23, count=1 << 24, load=1 << 25, ws=1 << 26, nb=1 << 20):
    return lib.tag_balance(Q, S, dtype, x, xs, mask, M, use, coef, grad, gs, acc, loss, count, load, ws, nb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(Q=0), EINVAL), (dict(S=0), EINVAL), (dict(S=16385, xs=20000, gs=20000), ESHAPE), (dict(dtype=3), EINVAL),
    (dict(M=0), EINVAL), (dict(M=65), EINVAL), (dict(coef=-1.0), EINVAL), (dict(coef=float("nan")), EINVAL),
    (dict(coef=float("inf")), EINVAL), (dict(x=None), EINVAL), (dict(mask=None), EINVAL), (dict(grad=None), EINVAL),
    (dict(loss=None), EINVAL), (dict(count=None), EINVAL), (dict(load=None), EINVAL), (dict(ws=None), EINVAL),
    (dict(xs=99), EINVAL), (dict(gs=99), EINVAL), (dict(dtype=1, acc=1), EINVAL), (dict(grad=(1 << 20) + 400), EINVAL),
    (dict(grad=(1 << 22) + 2), EINVAL), (dict(mask=(1 << 21) + 4), EINVAL), (dict(ws=(1 << 26) + 8), EINVAL),
    (dict(nb=100), ENOSPACE),
])
def test_balance_refuses(lib, kw, status):
    assert _balance(lib, **kw) == status
    assert lib.tag_last_error()


def test_scores_refuses_null_arguments(lib):
    assert lib.tag_gnn_scores(None, None, None, 1, None, None, None, 1, None, None, None, None, None, 0, None) == EINVAL


# ------------------------------------------------------------ the restatements
def test_gradient_restatement_is_the_loss_s_derivative():
    rng = np.random.default_rng(3)
    x = rng.normal(0, 1.5, (7, 12))
    masks = rng.integers(1, 1 << 5, 12).astype(np.uint64)
    use = np.array([1, 1, 0, 1, 1, 1, 1], bool)
    loss, grad, count, load, _ = R.balance(x, masks, 5, 0.3, use)
    assert abs(load.sum() - 1.0) < 1e-12 and count.sum() == 6
    num, d = np.zeros_like(x), 1e-6
    for i in np.ndindex(x.shape):
        hi, lo = x.copy(), x.copy()
        hi[i] += d
        lo[i] -= d
        num[i] = (R.balance_loss(hi, masks, 5, 0.3, use, load) - R.balance_loss(lo, masks, 5, 0.3, use, load)) / (2 * d)
    assert np.abs(num - grad).max() < 1e-8 and np.all(grad[2] == 0)


def test_even_decisions_have_the_least_loss():
    x = np.full((4, 4), -1e9)
    x[np.arange(4), np.arange(4)] = 0.0
    masks = np.array([1, 2, 4, 8], np.uint64)
    assert abs(R.balance(x, masks, 4, 0.25)[0] - 0.25) < 1e-12
    x[:, 0] = 10.0
    assert R.balance(x, masks, 4, 0.25)[0] > 0.9


def test_constrained_restatement_by_hand():
    x = np.array([[2.0, -2.0, 1.0, 0.5]], np.float32)
    y, _ = R.constrained(x, allow=np.array([[0b1011]], np.uint32), history=np.array([[0, 1, 1, 9, -1]]),
                         rep=np.array([2.0], np.float32), pre=np.array([0.25], np.float32),
                         frq=np.array([0.5], np.float32))
    assert y.tolist() == [[0.25, -5.25, -np.inf, 0.5]]
    p, at, best = R.priors(y)
    assert at[0] == 3 and best[0] == 0.5 and abs(p.sum() - 1) < 1e-12 and p[0, 2] == 0
    p, at, best = R.priors(np.full((1, 3), -np.inf))
    assert at[0] == -1 and np.isneginf(best[0]) and not p.any()
