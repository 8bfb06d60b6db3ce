"""The optimiser operators without a GPU: what their C entry points refuse before
anything is enqueued, and the 64-bit restatement that the GPU tests compare
with."""
import ctypes as C

import numpy as np
import pytest

from tests import _optim as R

EINVAL, ESHAPE, ENOSPACE = -1, -4, -5


@pytest.fixture(scope="module")
def abi():
    import paper_2302_06126_amd as P
    P._abi.load()
    return P._abi


def _ns(abi, steps=5, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7):
    return abi.tag_newton_schulz(steps, a, b, c, eps)


def _arr(abi, base, row, mat):
    return abi.tag_matrices(base, row, mat)


def _ortho(abi, count=2, rows=8, cols=6, x=(1 << 20, 6, 48), y=(1 << 24, 6, 48), n=1, dtype=0, ns=None, ws=1 << 28,
           nb=1 << 30):
    g = (abi.tag_ortho_group * 1)()
    g[0].count, g[0].rows, g[0].cols = count, rows, cols
    setattr(g[0], "in", _arr(abi, *x))
    g[0].out = _arr(abi, *y)
    return abi.load().tag_orthogonalise(g, n, dtype, C.byref(_ns(abi) if ns is None else ns), ws, nb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), EINVAL), (dict(count=0), EINVAL), (dict(rows=0), EINVAL), (dict(cols=0), EINVAL), (dict(dtype=2), EINVAL),
    (dict(rows=32769, x=(1 << 20, 6, 1 << 20), y=(1 << 24, 6, 1 << 20)), ESHAPE),
    (dict(count=1 << 20, rows=20000, cols=20000, x=(1 << 20, 20000, 1 << 30), y=(1 << 24, 20000, 1 << 30)), ESHAPE),
    # (launches of 2^32 threads and more)
    (dict(count=(1 << 19) + 1), ESHAPE),
    (dict(count=3, rows=32768, cols=32768, x=(1 << 20, 32768, 1 << 30), y=(1 << 50, 32768, 1 << 30)), ESHAPE),
    (dict(x=(None, 6, 48)), EINVAL), (dict(y=(None, 6, 48)), EINVAL), (dict(x=((1 << 20) + 2, 6, 48)), EINVAL),
    (dict(x=(1 << 20, 5, 48)), EINVAL), (dict(y=(1 << 24, 5, 48)), EINVAL), (dict(x=(1 << 20, 6, -48)), EINVAL),
    # results that overlap: a matrix stride of nothing, within a matrix, across interleaved rows
    (dict(y=(1 << 24, 6, 0)), EINVAL), (dict(y=(1 << 24, 6, 47)), EINVAL), (dict(y=(1 << 24, 11, 6)), EINVAL),
    (dict(ws=None), EINVAL), (dict(ws=(1 << 28) + 8), EINVAL), (dict(nb=1000), ENOSPACE),
])
def test_orthogonalise_refuses(abi, kw, status):
    assert _ortho(abi, **kw) == status
    assert abi.load().tag_last_error()


@pytest.mark.parametrize("kw", [dict(steps=0), dict(steps=33), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
                                dict(eps=float("inf")), dict(a=float("nan")), dict(c=float("inf")),
                                dict(a=5.0, b=0.0, c=0.0),            # grows without end
                                dict(a=1.0, b=16.0, c=-16.0),         # B leaves its range
                                dict(a=3.4445, b=-4.7750, c=4.0), dict(a=-4.0, b=0.0, c=0.0)])
def test_iterations_that_leave_the_range_are_refused(abi, kw):
    assert _ortho(abi, ns=_ns(abi, **kw)) == EINVAL
    assert abi.load().tag_last_error()


def test_iterations_of_every_length_in_range_pass_the_checks(abi):
    """(up to the workspace, which is too small)"""
    for kw in (dict(steps=1), dict(steps=32), dict(a=1.5, b=-0.5, c=0.0), dict(a=2.0, b=-1.5, c=0.5, steps=20),
               dict(a=1.0, b=0.0, c=0.0, steps=7)):
        assert _ortho(abi, ns=_ns(abi, **kw), nb=16) == ENOSPACE


def _muon(abi, count=2, rows=8, cols=6, plain=0, w=(1 << 20, 6, 48), g=(1 << 21, 6, 48), m=(1 << 22, 6, 48), n=1,
          lr=0.1, mu=0.9, wd=0.0, ws=1 << 28, nb=1 << 30, opt=True):
    q = (abi.tag_muon_group * 1)()
    q[0].count, q[0].rows, q[0].cols, q[0].plain = count, rows, cols, plain
    q[0].w, q[0].g, q[0].m = _arr(abi, *w), _arr(abi, *g), _arr(abi, *m)
    o = abi.tag_muon_options(lr, mu, wd, 1)
    return abi.load().tag_muon_step(q, n, C.byref(_ns(abi)), C.byref(o) if opt else None, ws, nb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), EINVAL), (dict(count=0), EINVAL), (dict(w=(None, 6, 48)), EINVAL), (dict(g=(None, 6, 48)), EINVAL),
    (dict(m=(None, 6, 48)), EINVAL), (dict(w=(1 << 21, 6, 48)), EINVAL), (dict(m=(1 << 21, 6, 48)), EINVAL),
    (dict(m=(1 << 20, 6, 48)), EINVAL), (dict(w=(1 << 20, 5, 48)), EINVAL), (dict(m=(1 << 22, 6, 0)), EINVAL),
    (dict(lr=-1.0), EINVAL), (dict(lr=float("nan")), EINVAL), (dict(lr=float("inf")), EINVAL), (dict(mu=1.0), EINVAL),
    (dict(mu=-0.1), EINVAL), (dict(wd=-1.0), EINVAL), (dict(wd=float("inf")), EINVAL), (dict(opt=False), EINVAL),
    (dict(nb=1000), ENOSPACE), (dict(ws=None), EINVAL),
])
def test_muon_refuses(abi, kw, status):
    assert _muon(abi, **kw) == status
    assert abi.load().tag_last_error()


def test_workspaces_hold_the_largest_set_of_groups(abi):
    lib = abi.load()
    g = (abi.tag_ortho_group * 40)()
    for i, q in enumerate(g):
        q.count, q.rows, q.cols = 1, 64, 64 * (1 + i)
    b, one = C.c_size_t(0), C.c_size_t(0)
    assert lib.tag_orthogonalise_workspace(g, 40, C.byref(b)) == 0
    # sets of groups run one after the other in the same workspace: it holds the largest group, and not all of them
    sizes = []
    for i in range(40):
        part = C.cast(C.byref(g[i]), C.POINTER(abi.tag_ortho_group))
        assert lib.tag_orthogonalise_workspace(part, 1, C.byref(one)) == 0
        sizes.append(one.value)
    assert max(sizes) < b.value < sum(sizes) and max(sizes) > 16 * 64 * 64 * 40
    assert lib.tag_orthogonalise_workspace(g, 40, None) == EINVAL
    assert lib.tag_orthogonalise_workspace(None, 1, C.byref(b)) == EINVAL
    q = (abi.tag_muon_group * 1)()
    q[0].count, q[0].rows, q[0].cols, q[0].plain = 1, 1, 100000, 1
    assert lib.tag_muon_workspace(q, 1, C.byref(b)) == 0 and b.value == 0
    q[0].plain = 0
    assert lib.tag_muon_workspace(q, 1, C.byref(b)) == ESHAPE


# ------------------------------------------------------------ the restatement
@pytest.mark.parametrize("shape", [(8, 8), (64, 300), (90, 40)])
def test_restatement_with_the_bf16_forms_roundings(shape):
    """Near the exact one (2^-11 of an operand's elements, five steps), and not equal to it."""
    g = np.random.default_rng(shape).normal(0, 1, shape)
    want = R.newton_schulz(g)[0]
    err = np.linalg.norm(R.rounded_bf16(g) - want) / np.linalg.norm(want)
    assert 1e-5 < err < 2.0 ** -8


@pytest.mark.parametrize("shape", [(5, 9), (9, 5), (16, 16), (1, 7)])
def test_restatement_is_the_iteration_of_products(shape):
    g = np.random.default_rng(shape).normal(0, 1, shape)
    want, _ = R.newton_schulz(g)
    x = g if shape[0] <= shape[1] else g.T
    x = x / (np.linalg.norm(x) + 1e-7)
    a, b, c = R.QUINTIC
    for _ in range(5):
        A = x @ x.T
        x = a * x + (b * A + c * A @ A) @ x
    x = x if shape[0] <= shape[1] else x.T
    assert np.abs(x - want).max() < 1e-12
    s = np.linalg.svd(want, compute_uv=False)
    assert s.max() < 1.3
