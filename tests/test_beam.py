"""Beam search without a GPU: what the C entry points refuse before anything is
enqueued, and the restatement that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest

from tests import _beam as R

EINVAL, ESHAPE, ENOSPACE = -1, -4, -5


@pytest.fixture(scope="module")
def lib():
    import paper_2302_06126_amd as P
    return P._abi.load()


def _select(lib, n=2, V=3, W=4, S=10, dtype=0, x=1 << 20, xs=10, tin=1 << 21, done=None, total=1 << 22, parent=1 << 23,
            slice_=1 << 24, ws=1 << 25, nb=1 << 30):
    return lib.tag_beam_select(n, V, W, S, dtype, x, xs, tin, done, total, parent, slice_, ws, nb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), EINVAL), (dict(V=0), EINVAL), (dict(W=0), EINVAL), (dict(S=0), EINVAL), (dict(V=257), ESHAPE),
    (dict(W=257), ESHAPE), (dict(n=1 << 22), ESHAPE), (dict(V=256, S=(1 << 22) + 1, xs=1 << 23), ESHAPE),
    (dict(dtype=2), EINVAL), (dict(x=None), EINVAL), (dict(tin=None), EINVAL), (dict(total=None), EINVAL),
    (dict(parent=None), EINVAL), (dict(slice_=None), EINVAL), (dict(xs=9), EINVAL), (dict(x=(1 << 20) + 2), EINVAL),
    (dict(dtype=1, x=(1 << 20) + 1), EINVAL), (dict(tin=(1 << 21) + 1), EINVAL), (dict(parent=(1 << 23) + 2), EINVAL),
    # outputs on inputs or on one another
    (dict(total=1 << 21), EINVAL),                    # (widths differ)
    (dict(V=4, total=(1 << 21) + 4), EINVAL), (dict(parent=(1 << 20) + 40), EINVAL), (dict(slice_=1 << 21), EINVAL),
    (dict(done=(1 << 22) + 30), EINVAL), (dict(parent=1 << 22), EINVAL), (dict(slice_=(1 << 23) + 28), EINVAL),
])
def test_select_refuses(lib, kw, status):
    assert _select(lib, **kw) == status
    assert lib.tag_last_error()


def test_no_searches_are_nothing(lib):
    assert _select(lib, n=0, x=None, tin=None, total=None) == 0
    assert lib.tag_beam_reorder(0, 4, 4, None, None, 0, None) == 0
    assert lib.tag_beam_reorder(3, 4, 4, None, None, 0, None) == 0


def test_workspace(lib):
    b = C.c_size_t(7)
    assert lib.tag_beam_workspace(1, 4, 4, 60, C.byref(b)) == 0
    assert lib.tag_beam_workspace(8, 256, 256, 1 << 22, C.byref(b)) == 0
    assert lib.tag_beam_workspace(1, 4, 4, 0, C.byref(b)) == EINVAL
    assert lib.tag_beam_workspace(1, 4, 257, 60, C.byref(b)) == ESHAPE
    assert lib.tag_beam_workspace(1, 4, 4, 60, None) == EINVAL


def _reorder(lib, states, n=2, V=4, W=4, parent=1 << 12, n_states=None):
    from paper_2302_06126_amd._abi import tag_beam_state
    arr = (tag_beam_state * max(len(states), 1))(*[tag_beam_state(*s) for s in states])
    return lib.tag_beam_reorder(n, V, W, parent, arr, len(states) if n_states is None else n_states, None)


A, B = 1 << 20, 1 << 24


@pytest.mark.parametrize("states,kw,status", [
    ([(A, B, 10, 40, 10, 40, 10)], dict(W=0), EINVAL), ([(A, B, 10, 40, 10, 40, 10)], dict(V=300), ESHAPE),
    ([(A, B, 10, 40, 10, 40, 10)], dict(n_states=65), EINVAL), ([(A, B, 10, 40, 10, 40, 10)], dict(n_states=-1), EINVAL),
    ([(A, B, 10, 40, 10, 40, 10)], dict(parent=None), EINVAL), ([(A, B, 10, 40, 10, 40, 10)], dict(parent=4097), EINVAL),
    ([(A, B, -1, 40, 10, 40, 10)], {}, EINVAL), ([(None, B, 10, 40, 10, 40, 10)], {}, EINVAL),
    ([(A, None, 10, 40, 10, 40, 10)], {}, EINVAL), ([(A, B, 10, -40, 10, 40, 10)], {}, EINVAL),
    ([(A, B, 10, 40, 10, 40, -10)], {}, EINVAL),
    ([(A, B, 10, 40, 10, 40, 9)], {}, EINVAL),                   # rows of out overlap
    ([(A, B, 10, 40, 10, 39, 10)], {}, EINVAL), ([(A, B, 10, 40, 10, 0, 10)], {}, EINVAL),
    ([(A, A, 10, 40, 10, 48, 12)], {}, EINVAL),                  # in place with other strides
    ([(A, A, 10, 40, 10, 40, 10)], dict(V=6), EINVAL),           # in place, searches overlap at the larger width
    ([(A, A + 10, 10, 40, 10, 40, 10)], {}, EINVAL), ([(A, A + 5, 10, 80, 20, 80, 20)], {}, EINVAL),
    ([(A, B, 10, 40, 10, 40, 10), (A + 100, B + 79, 10, 40, 10, 40, 10)], {}, EINVAL),   # outs meet
    ([(A, B, 10, 40, 10, 40, 10), (B + 79, B + 400, 10, 40, 10, 40, 10)], {}, EINVAL),   # an out on another's in
    ([(A, B, 10, 40, 10, 40, 10)], dict(parent=B + 76), EINVAL),
    # (launches of 2^32 threads and more; sizes whose products leave 64 bits)
    ([(A, 1 << 61, 1 << 30, 1 << 32, 1 << 30, 1 << 32, 1 << 30)], dict(n=1 << 10), ESHAPE),
    ([(A, 1 << 61, 1 << 40, 1 << 45, 1 << 40, 1 << 45, 1 << 40)], dict(n=(1 << 31) - 1), ESHAPE),
    ([(A, 1 << 61, 1 << 45, 0, 0, 1 << 45, 0)], dict(n=3, W=1), ESHAPE),
    ([(A, B, 1 << 47, 0, 0, 0, 0)], dict(n=1, W=1), ESHAPE),
])
def test_reorder_refuses(lib, states, kw, status):
    assert _reorder(lib, states, **kw) == status
    assert lib.tag_last_error()


def test_objects_refuse_on_the_host():
    import torch
    from paper_2302_06126_amd import policy
    with pytest.raises(ValueError):
        policy.Reorder([torch.zeros(4, 3)], 1, 4)
    with pytest.raises(ValueError):
        policy.Reorder([], 1, 4)
    with pytest.raises(ValueError):
        policy.Beam(1, 4, 10, device="cpu")


# ------------------------------------------------------------ the restatement
def test_restatement_of_a_level_by_hand():
    x = np.log(np.array([[[0.5, 0.25, 0.25], [0.1, 0.2, 0.7]]]))
    t = np.log(np.array([[0.6, 0.4]]))
    total, parent, slice_, _ = R.select(x + 3.0, t, np.zeros((1, 2), bool), 3)   # (a shift of a row changes nothing)
    assert np.allclose(np.exp(total), [[0.3, 0.28, 0.15]])
    assert parent.tolist() == [[0, 1, 0]] and slice_.tolist() == [[0, 2, 1]]
    total, parent, slice_, _ = R.select(x, t, np.array([[False, True]]), 3)
    assert np.allclose(np.exp(total), [[0.4, 0.3, 0.15]]) and parent.tolist() == [[1, 0, 0]]
    assert slice_.tolist() == [[-1, 0, 1]]


def test_restatement_is_the_best_of_all_paths():
    """Three levels of a search as wide as there are paths: every path's probability."""
    rng = np.random.default_rng(4)
    S, total = 3, np.array([[0.0]])
    tables = rng.normal(0, 1, (3, S, S))          # level, last slice, next slice
    paths = [[()]]
    for level in range(3):
        V = total.shape[1]
        x = np.stack([tables[level, p[-1] if p else 0] for p in paths[0]])[None]
        total, parent, slice_, _ = R.select(x, total, np.zeros((1, V), bool), V * S)
        paths = [[paths[0][v] + (int(a),) for v, a in zip(parent[0], slice_[0])]]
    assert len(set(paths[0])) == S ** 3 and abs(np.exp(total).sum() - 1.0) < 1e-12
    p = lambda t: t - np.log(np.exp(t).sum())
    for path, lp in zip(paths[0], total[0]):
        want = p(tables[0, 0])[path[0]] + p(tables[1, path[0]])[path[1]] + p(tables[2, path[1]])[path[2]]
        assert abs(want - lp) < 1e-12


def test_restatement_drops_what_has_no_probability():
    x = np.zeros((1, 5, 2))
    x[0, 0, 1] = np.nan
    x[0, 1, 0] = np.inf
    x[0, 2] = -np.inf
    x[0, 3, 0] = -np.inf
    t = np.array([[0.0, 0.0, 0.0, -1.0, np.nan]])
    total, parent, slice_, _ = R.select(x, t, np.zeros((1, 5), bool), 3)
    assert total[0].tolist() == [-1.0, -np.inf, -np.inf] and parent[0].tolist() == [3, -1, -1]
    assert slice_[0].tolist() == [1, -1, -1]
