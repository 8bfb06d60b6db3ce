"""Arrays of one group that share elements, without a GPU: a result that stands on
part of its input (a block would read what another has written) and a weight,
gradient or momentum on part of another are refused, arrays that only interleave
are not.  A call that passes its checks ends at the workspace, which is too small."""
import ctypes as C

import numpy as np
import pytest

EINVAL, ENOSPACE = -1, -5
BASE = 1 << 20


@pytest.fixture(scope="module")
def abi():
    import paper_2302_06126_amd as P
    P._abi.load()
    return P._abi


def _ortho(abi, shape, x, y, dtype=0):
    """x, y: (offset in elements, row stride, matrix stride)"""
    el = 2 if dtype else 4
    g = (abi.tag_ortho_group * 1)()
    g[0].count, g[0].rows, g[0].cols = shape
    setattr(g[0], "in", abi.tag_matrices(BASE + el * x[0], *x[1:]))
    g[0].out = abi.tag_matrices(BASE + el * y[0], *y[1:])
    ns = abi.tag_newton_schulz(5, 3.4445, -4.7750, 2.0315, 1e-7)
    return abi.load().tag_orthogonalise(g, 1, dtype, C.byref(ns), 1 << 28, 16, None)


def _muon(abi, shape, *arrays, plain=0):
    g = (abi.tag_muon_group * 1)()
    g[0].count, g[0].rows, g[0].cols, g[0].plain = shape + (plain,)
    g[0].w, g[0].g, g[0].m = (abi.tag_matrices(BASE + 4 * a[0], *a[1:]) for a in arrays)
    ns = abi.tag_newton_schulz(5, 3.4445, -4.7750, 2.0315, 1e-7)
    o = abi.tag_muon_options(0.1, 0.9, 0.0, 1)
    return abi.load().tag_muon_step(g, 1, C.byref(ns), C.byref(o), 1 << 28, 16, None)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape,x,y,status", [
    ((4, 8, 6), (0, 6, 48), (0, 6, 48), ENOSPACE),            # in place
    ((4, 8, 6), (0, 6, 48), (48, 6, 48), EINVAL),             # a matrix further on
    ((4, 8, 6), (48, 6, 48), (0, 6, 48), EINVAL),
    ((4, 8, 6), (0, 6, 48), (192, 6, 48), ENOSPACE),          # behind the last
    ((1, 8, 6), (0, 6, 0), (6, 6, 0), EINVAL),                # a row further on
    ((1, 8, 6), (0, 6, 0), (1, 6, 0), EINVAL),
    ((1, 8, 6), (0, 6, 0), (0, 7, 0), EINVAL),                # in place, other rows
    ((4, 8, 6), (0, 6, 48), (0, 24, 6), EINVAL),              # in place, matrices interleaved
    ((4, 8, 6), (0, 12, 96), (6, 12, 96), ENOSPACE),          # the two halves of wider rows
    ((4, 8, 6), (0, 12, 96), (5, 12, 96), EINVAL),
    ((4, 8, 6), (0, 24, 6), (24, 24, 6), EINVAL),             # rows of all matrices in turn, a row further on
    ((1, 1, 6), (0, 6, 0), (0, 99, 7), ENOSPACE),             # (strides that mean nothing)
    ((1, 1, 6), (0, 6, 0), (5, 99, 7), EINVAL),
    ((1, 1, 6), (0, 6, 0), (6, 99, 7), ENOSPACE),
])
def test_results_on_their_input(abi, shape, x, y, status, dtype):
    assert _ortho(abi, shape, x, y, dtype) == status


@pytest.mark.parametrize("shape,w,g,m,status", [
    ((1, 1, 100), (0, 100, 0), (100, 100, 0), (200, 100, 0), ENOSPACE),
    ((1, 1, 100), (0, 100, 0), (50, 100, 0), (200, 100, 0), EINVAL),
    ((1, 1, 100), (0, 100, 0), (100, 100, 0), (199, 100, 0), EINVAL),
    ((1, 1, 100), (0, 100, 0), (300, 100, 0), (99, 100, 0), EINVAL),
    ((3, 8, 6), (0, 18, 144), (6, 18, 144), (12, 18, 144), ENOSPACE),
    ((3, 8, 6), (0, 18, 144), (6, 18, 144), (13, 18, 144), EINVAL),
])
def test_arrays_of_a_step(abi, shape, w, g, m, status):
    assert _muon(abi, shape, w, g, m) == status


def test_against_the_elements_themselves(abi):
    rng = np.random.default_rng(2302)
    seen = set()
    for _ in range(400):
        count, rows, cols = (int(v) for v in rng.integers(1, 5, 3))
        row, mat = cols + int(rng.integers(0, 4)), int(rng.integers(0, 30))
        at = (np.arange(count)[:, None, None] * mat + np.arange(rows)[:, None] * row + np.arange(cols)).ravel()
        if len(set(at)) < len(at):   # (refused for itself)
            continue
        d = int(rng.integers(-at.max() - 3, at.max() + 4))
        if d == 0:
            continue
        want = EINVAL if set(at) & set(at + d) else ENOSPACE
        got = _ortho(abi, (count, rows, cols), (500, row, mat), (500 + d, row, mat))
        span = (rows - 1) * row + cols
        if count > 1 and mat < span and not (mat >= cols and (rows == 1 or row >= (count - 1) * mat + cols)):
            assert got == EINVAL     # (interleaving that the entry point does not know)
            continue
        assert got == want, (count, rows, cols, row, mat, d)
        seen.add(want)
    assert seen == {EINVAL, ENOSPACE}
