"""Clipping by the global norm without a GPU: what the C entry points and the
objects refuse before anything is enqueued, and how tensors are taken apart."""
import ctypes as C

import numpy as np
import pytest

EINVAL, ESHAPE, ENOSPACE = -1, -4, -5
A, B = 1 << 20, 1 << 30


@pytest.fixture(scope="module")
def lib():
    import paper_2302_06126_amd as P
    return P._abi.load()


def _bytes(lib, arrays, n=None):
    from paper_2302_06126_amd._abi import tag_clip_array
    arr = (tag_clip_array * max(len(arrays), 1))(*[tag_clip_array(*a) for a in arrays])
    b = C.c_size_t(0)
    st = lib.tag_clip_table_bytes(arr, len(arrays) if n is None else n, C.byref(b))
    return st, b.value


@pytest.mark.parametrize("arrays,status", [
    ([(None, B, 1, 4, 4, 4, 0)], EINVAL), ([(A, B, -1, 4, 4, 4, 0)], EINVAL), ([(A, B, 1, -4, 4, 4, 0)], EINVAL),
    ([(A, B, 1, 4, 4, 4, 2)], EINVAL), ([(A + 2, B, 1, 4, 4, 4, 0)], EINVAL), ([(A, B + 1, 1, 4, 4, 4, 1)], EINVAL),
    ([(A, B, 3, 4, 3, 4, 0)], EINVAL), ([(A, B, 3, 4, 4, 3, 0)], EINVAL), ([(A, A, 3, 4, 4, 5, 0)], EINVAL),
    ([(A, A + 8, 1, 4, 4, 4, 0)], EINVAL), ([(A, A + 8, 3, 4, 5, 5, 0)], EINVAL),
    # outputs on other arrays, the same gradient in place twice or once in place and once for the norm alone
    ([(A, A, 1, 4, 4, 4, 0), (A + 16, A + 12, 1, 1, 1, 1, 0)], EINVAL),
    ([(A, B, 1, 4, 4, 4, 0), (A + 64, B + 12, 1, 4, 4, 4, 0)], EINVAL),
    ([(A, A, 1, 4, 4, 4, 0), (A, A, 1, 4, 4, 4, 0)], EINVAL), ([(A, A, 1, 4, 4, 4, 0), (A, None, 1, 4, 4, 4, 0)], EINVAL),
    ([(A, None, 1 << 45, 1, 1, 1, 0)], ESHAPE), ([(A, None, 1 << 30, 1 << 30, 1 << 30, 0, 0)], ESHAPE),
    ([(A, None, 1, 1 << 40, 1 << 40, 0, 0)], ESHAPE), ([(A, None, 4, 3, 1 << 60, 0, 0)], ESHAPE),
])
def test_arrays_are_refused(lib, arrays, status):
    assert _bytes(lib, arrays)[0] == status
    assert lib.tag_last_error()


def test_table_sizes(lib):
    assert _bytes(lib, []) == (0, 0) and _bytes(lib, [], n=-1)[0] == EINVAL
    one = _bytes(lib, [(A, None, 1, 1, 1, 0, 0)])[1]
    assert one == 64
    assert _bytes(lib, [(A, None, 0, 5, 5, 0, 0), (A, None, 5, 0, 5, 0, 0), (None, None, 0, 0, 0, 0, 0)]) == (0, 0)
    # 4096 fp32 or 8192 bf16 values to an entry; wide rows have entries of their own, narrow ones share them
    assert _bytes(lib, [(A, B, 1, 4097, 1, 1, 0)])[1] == 2 * one and _bytes(lib, [(A, B, 1, 8192, 1, 1, 1)])[1] == one
    assert _bytes(lib, [(A, B, 3, 1024, 1025, 1024, 0)])[1] == 3 * one
    assert _bytes(lib, [(A, B, 25, 40, 41, 40, 0)])[1] == one and _bytes(lib, [(A, B, 26, 40, 41, 40, 0)])[1] == 2 * one
    # parts of wider rows, side by side, in place; vectors side by side, each into another's neighbour
    assert _bytes(lib, [(A, A, 8, 10, 30, 30, 0), (A + 40, A + 40, 8, 20, 30, 30, 0)])[0] == 0
    assert _bytes(lib, [(A, B, 1, 4, 4, 4, 0), (A + 16, B + 16, 1, 4, 4, 4, 0)])[0] == 0
    assert _bytes(lib, [(A, A, 8, 10, 30, 30, 0), (A + 40, A + 40, 8, 21, 30, 30, 0)])[0] == EINVAL
    # the same gradient twice for the norm alone
    assert _bytes(lib, [(A, None, 1, 4, 4, 0, 0), (A, None, 1, 4, 4, 0, 0)])[0] == 0


def test_calls_are_refused(lib):
    from paper_2302_06126_amd._abi import tag_clip_array, tag_clip_plan
    arr = (tag_clip_array * 1)(tag_clip_array(A, B, 1, 5000, 5000, 5000, 0))
    plan = tag_clip_plan()
    assert lib.tag_clip_table_bytes(arr, 1, None) == EINVAL
    assert lib.tag_clip_prepare(arr, 1, 4096, 128, None, None) == EINVAL
    assert lib.tag_clip_prepare(arr, 1, 4096, 127, None, C.byref(plan)) == ENOSPACE
    assert lib.tag_clip_prepare(arr, 1, None, 128, None, C.byref(plan)) == EINVAL
    assert lib.tag_clip_prepare(arr, 1, 4097, 128, None, C.byref(plan)) == EINVAL
    b = C.c_size_t(0)
    assert lib.tag_clip_workspace(C.byref(b)) == 0 and lib.tag_clip_workspace(None) == EINVAL
    plan = tag_clip_plan(4096, 2, 1)
    call = lambda p=plan, limit=1.0, result=8192, ws=1 << 20, nb=b.value: lib.tag_clip(
        C.byref(p) if p else None, limit, result, ws, nb, None)
    for bad, st in ((dict(p=None), EINVAL), (dict(result=None), EINVAL), (dict(limit=-1.0), EINVAL),
                    (dict(limit=float("nan")), EINVAL), (dict(result=8193), EINVAL), (dict(ws=None), EINVAL),
                    (dict(ws=(1 << 20) + 8), EINVAL), (dict(nb=b.value - 1), ENOSPACE),
                    (dict(p=tag_clip_plan(None, 2, 1)), EINVAL), (dict(p=tag_clip_plan(4096, -1, 1)), EINVAL),
                    (dict(p=tag_clip_plan(4096, 2, 3)), EINVAL)):
        assert call(**bad) == st, bad


def test_objects_refuse_on_the_host():
    import torch
    from paper_2302_06126_amd import optim
    with pytest.raises(ValueError):
        optim.Clip([], 1.0)
    with pytest.raises(ValueError):
        optim.Clip([torch.zeros(3)], 1.0)


@pytest.mark.parametrize("seed", range(6))
def test_tensors_are_taken_apart(seed):
    """The pieces address every element once, g's and out's alike."""
    import torch
    from paper_2302_06126_amd.optim import _pieces
    rng = np.random.default_rng(seed)
    base = torch.arange(6 * 7 * 8 * 9, dtype=torch.float32).view(6, 7, 8, 9)
    views = [base, base[1:, 2:, 3:, 4:], base[:, :, ::2], base[:, 1:, :, :5], base[2, 3, 4], base[2, :, 3, 1], base[0, 0, 0, :1],
             base[:, :1], base[::2, :, :, 1:2], base.view(6, -1)[:, 5:77], base[3, 3, 3, 3]]
    for v in views:
        out = torch.zeros([s + int(rng.integers(0, 2)) for s in v.shape])[tuple(slice(0, s) for s in v.shape)]
        seen = {}
        for g, y, rows, cols, gs, os in _pieces(v, out):
            for r in range(rows):
                for c in range(cols):
                    a, b = (g - base.data_ptr()) // 4 + r * gs + c, (y - out.data_ptr()) // 4 + r * os + c
                    assert a not in seen
                    seen[a] = b
        offsets = lambda t, o: sorted((int(sum(i * s for i, s in zip(ix, t.stride()))) + o, ix) for ix in np.ndindex(*t.shape))
        at = {ix: b for b, ix in offsets(out, 0)}
        want = {a: at[ix] for a, ix in offsets(v, v.storage_offset())}
        assert seen == want, v.shape
    with pytest.raises(ValueError):
        _pieces(base[0, 0].t(), None)
