"""The optimiser step from clipped gradients without a GPU: its refusals, and the
step's options as C programs that know nothing of it lay them out.  A call that
passes its checks ends at the workspace, which is too small."""
import ctypes as C

import pytest

EINVAL, ENOSPACE = -1, -5
W, G, M, CLIP = 1 << 20, 1 << 22, 1 << 24, 1 << 26


@pytest.fixture(scope="module")
def abi():
    import paper_2302_06126_amd as P
    P._abi.load()
    return P._abi


def _group(abi, count=1, rows=70, cols=90, row=90, mat=0):
    g = (abi.tag_muon_group * 1)()
    g[0].count, g[0].rows, g[0].cols = count, rows, cols
    g[0].w, g[0].g, g[0].m = (abi.tag_matrices(p, row, mat) for p in (W, G, M))
    return g, abi.tag_newton_schulz(5, 3.4445, -4.7750, 2.0315, 1e-7)


@pytest.mark.parametrize("behind", [0, 3, 2 ** 64 - 1])
def test_options_are_their_four_fields(abi, behind):
    """Whatever stands behind them is not looked at."""
    options = (C.c_float * 4)(0.1, 0.9, 0.0, 0.0)
    raw = (C.c_uint8 * 24).from_buffer_copy(bytes(options) + behind.to_bytes(8, "little"))
    g, ns = _group(abi)
    step = abi.load().tag_muon_step
    assert step(g, 1, C.byref(ns), C.cast(raw, C.POINTER(abi.tag_muon_options)), 1 << 28, 16, None) == ENOSPACE
    assert C.sizeof(abi.tag_muon_options) == 16


def _clipped(abi, clip=CLIP, options=True, ws=1 << 28, nb=16, **kw):
    g, ns = _group(abi, **kw)
    o = abi.tag_muon_options(0.1, 0.9, 0.0, 1)
    return abi.load().tag_muon_step_clipped(g, 1, C.byref(ns), C.byref(o) if options else None, clip, ws, nb, None)


WIDE = dict(count=3, rows=70, cols=90, row=100, mat=7000)


@pytest.mark.parametrize("kw,status", [
    (dict(), ENOSPACE), (dict(clip=None), EINVAL), (dict(clip=CLIP + 2), EINVAL), (dict(options=False), EINVAL),
    # among weights or momentum, which the step writes while it looks at them; beside them; among the gradients
    (dict(clip=W), EINVAL), (dict(clip=M), EINVAL), (dict(clip=W + 4 * (70 * 90 - 1)), EINVAL), (dict(clip=M - 4), EINVAL),
    (dict(clip=W - 8), ENOSPACE), (dict(clip=W + 4 * 70 * 90), ENOSPACE), (dict(clip=G), ENOSPACE),
    # and between their rows and matrices
    (dict(clip=W + 4 * 92, **WIDE), ENOSPACE), (dict(clip=W + 4 * 89, **WIDE), EINVAL),
    (dict(clip=W + 4 * 99, **WIDE), EINVAL), (dict(clip=W + 4 * (7000 + 6 * 100 + 90), **WIDE), ENOSPACE),
    (dict(clip=M + 4 * (14000 + 69 * 100 + 89), **WIDE), EINVAL), (dict(clip=M + 4 * (14000 + 69 * 100 + 90), **WIDE), ENOSPACE),
])
def test_clipped_step_refuses(abi, kw, status):
    assert _clipped(abi, **kw) == status
    assert abi.load().tag_last_error()


def test_clip_in_another_group(abi):
    g, ns = _group(abi)
    two = (abi.tag_muon_group * 2)(g[0], g[0])
    two[1].w.base, two[1].m.base = CLIP - 4 * 90, 1 << 27
    two[1].plain = 1
    o = abi.tag_muon_options(0.1, 0.9, 0.0, 1)
    step = abi.load().tag_muon_step_clipped
    assert step(two, 2, C.byref(ns), C.byref(o), CLIP, 1 << 28, 16, None) == EINVAL
    assert step(two, 2, C.byref(ns), C.byref(o), 1 << 30, 1 << 28, 16, None) == ENOSPACE
