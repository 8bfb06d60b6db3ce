"""fp32 matrices and optimiser steps against the iteration in 64 bits, to the bound
that products with a lost or exchanged part do not keep (_split.BOUND,
test_optim_split.py), at every size at which the kernels' form changes."""
import numpy as np
import pytest

from tests import _optim as R
from tests import _split as S
from tests.test_optim_split import gradient

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _near(got, g, what, rounded=0.0):
    """rounded: of the result's norm, what its own fp32 operations cost."""
    want = R.newton_schulz(g)[0]
    err = np.linalg.norm(np.asarray(got, np.float64) - want) / np.linalg.norm(want)
    print(f"   {what} {g.shape}: {err:.2e}", flush=True)
    assert err <= S.BOUND + rounded


@pytest.mark.parametrize("count,shape", [
    (1, (3, 5)), (1, (31, 33)), (2, (64, 64)), (1, (64, 128)), (1, (200, 64)), (3, (64, 256)), (1, (256, 7)),   # one launch
    (1, (1, 300)), (1, (65, 64)), (2, (100, 516)), (1, (257, 130)), (1, (64, 257)), (1, (400, 400)),           # tiles of 64
    (1, (129, 700)), (1, (700, 129)), (1, (1024, 1024)), (3, (900, 700)), (2, (520, 2100)), (40, (70, 130))])  # and of 128
def test_orthogonalise(torch, count, shape):
    from paper_2302_06126_amd.optim import orthogonalise
    g = np.stack([gradient(i, *shape) for i in range(count)])
    got = orthogonalise(torch.from_numpy(g).cuda()).cpu().numpy()
    for i in sorted({0, count - 1}):
        _near(got[i], g[i], "matrix")


@pytest.mark.parametrize("kind", ["equal", "normal", "orthogonal", "repeated"])
def test_other_matrices(torch, kind):
    from paper_2302_06126_amd.optim import orthogonalise
    rng = np.random.default_rng(13)
    g = {"equal": np.full((300, 300), 0.37), "normal": rng.normal(0, 1, (300, 900)),
         "orthogonal": np.linalg.qr(rng.normal(0, 1, (300, 300)))[0],
         "repeated": np.repeat(rng.normal(0, 1, (30, 900)), 10, axis=0)}[kind].astype(np.float32)
    _near(orthogonalise(torch.from_numpy(g).cuda()).cpu().numpy(), g, kind)


@pytest.mark.parametrize("shapes", [[(1, 64, 42), (2, 30, 200)], [(9, 128, 256), (128, 42), (128, 260)], [(12, 256, 512)],
                                    [(1, 1024, 1030), (300, 40)]])
def test_the_update_of_weights_at_zero(torch, shapes):
    """w = -lr factor O(u) with nothing to hide it: one product and a difference
    with zero are rounded, and lr and the factor themselves (4 half steps); u is
    rounded three times on its way, each like a relative error of its matrix, which
    the five steps raise by at most 3.4445^5 < 2^9 of the norm (2 such half steps
    of the norm's root mean square: 2^-15)."""
    from paper_2302_06126_amd.optim import Muon
    W = [torch.zeros(s, device="cuda") for s in shapes]
    gs = [np.stack([gradient(7 + i, *s[-2:]) for i in range(int(np.prod(s[:-2], dtype=int)))]).reshape(s) for s in shapes]
    ms = [np.stack([gradient(90 + i, *s[-2:]) for i in range(int(np.prod(s[:-2], dtype=int)))]).reshape(s) for s in shapes]
    G, M = ([torch.from_numpy(v).cuda() for v in vs] for vs in (gs, ms))
    Muon(list(zip(W, G)), lr=0.5, momentum=0.9, state=M).step()
    mu = np.float64(np.float32(0.9))
    for s, w, g, m in zip(shapes, W, gs, ms):
        u = (g + mu * (mu * m.astype(np.float64) + g)).reshape((-1,) + s[-2:])
        o = w.cpu().numpy().astype(np.float64).reshape(u.shape) / (-0.5 * np.sqrt(max(1.0, s[-2] / s[-1])))
        for i in sorted({0, len(u) - 1}):
            _near(o[i], u[i], "update", rounded=2.0 ** -15)
