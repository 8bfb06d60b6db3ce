"""Plain groups (momentum SGD) of the optimiser step, against the update in 64
bits.  m rounds a product and a sum at once, u the same, w two products and their
difference: in units of 2^-24, 1 of m, 2 of u (m's and its own), and 1 of w, 1 of
keep w (keep itself 1 more), 1 of lr u with u's 2 and lr's own."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _check(torch, w, m, w0, g, m0, lr=0.02, mu=0.95, wd=0.01, nesterov=True):
    """w, m after one step from w0, m0 (device tensors)."""
    lr, mu, wd = (float(np.float32(v)) for v in (lr, mu, wd))
    w0, g, m0 = w0.double(), g.double(), m0.double()
    m1 = mu * m0 + g
    size = m0.abs() + g.abs()
    assert bool(((m.double() - m1).abs() <= EPS * 2 * size).all())
    u = g + mu * m1 if nesterov else m1
    w1 = (1 - lr * wd) * w0 - lr * u
    assert bool(((w.double() - w1).abs() <= EPS * (4 * w0.abs() + 8 * lr * 2 * size)).all())


def _arrays(torch, n, seed=1):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    r = lambda s: s * torch.randn(n, generator=gen, device="cuda")
    return r(0.1), r(1e-3), r(1e-3)


def test_a_vector_of_more_than_2_25_elements(torch):
    from paper_2302_06126_amd.optim import Muon
    w, g, m = _arrays(torch, 2 ** 25 + 5)
    w0, m0 = w.clone(), m.clone()
    Muon([(w, g)], lr=0.02, weight_decay=0.01, state=[m]).step()
    _check(torch, w, m, w0, g, m0)


@pytest.mark.parametrize("n", [1, 3, 4095, 4096, 4097, 4100, 8191, 8192, 100003])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_vectors_of_whole_blocks_and_their_ends(torch, n, offset):
    """On either side of a block of 4,096 elements, rows that start between two
    accesses of four, and what lies around them."""
    from paper_2302_06126_amd.optim import Muon
    big = [v for v in _arrays(torch, n + 8, seed=n)]
    was = [v.clone() for v in big]
    w, g, m = (v[offset:offset + n] for v in big)
    for nesterov in (True, False):
        w0, m0 = w.clone(), m.clone()
        Muon([(w, g)], lr=0.02, weight_decay=0.01, state=[m], nesterov=nesterov).step()
        _check(torch, w, m, w0, g, m0, nesterov=nesterov)
    for v, k in zip(big, was):
        assert torch.equal(v[:offset], k[:offset]) and torch.equal(v[offset + n:], k[offset + n:])
    assert torch.equal(big[1], was[1])


@pytest.mark.parametrize("count,rows,cols,row,mat", [
    (3, 1, 5000, 5000, 5000), (3, 1, 5000, 5000, 5008), (2, 1, 4096, 4096, 4097), (2, 70, 60, 60, 4200),
    (2, 70, 60, 64, 4500), (3, 9, 1000, 1003, 9100), (1, 4097, 1, 1, 4097), (1, 4097, 1, 3, 12291), (4, 6, 700, 2800, 700)])
def test_plain_groups_of_rows(torch, count, rows, cols, row, mat):
    """By the C entry point: several matrices, several rows, rows and matrices
    apart, interleaved ones, and the padding between them."""
    import ctypes as C
    import paper_2302_06126_amd as P
    from paper_2302_06126_amd._abi import (check, tag_matrices, tag_muon_group, tag_muon_options, tag_newton_schulz)
    n = (count - 1) * mat + (rows - 1) * row + cols + 7
    w, g, m = _arrays(torch, n, seed=rows)
    at = (np.arange(count)[:, None, None] * mat + np.arange(rows)[:, None] * row + np.arange(cols)).ravel()
    at = torch.from_numpy(at).cuda()
    w0, g0, m0 = w.clone(), g.clone(), m.clone()
    q = (tag_muon_group * 1)()
    q[0].count, q[0].rows, q[0].cols, q[0].plain = count, rows, cols, 1
    q[0].w, q[0].g, q[0].m = (tag_matrices(t.data_ptr(), row, mat) for t in (w, g, m))
    ns, o = tag_newton_schulz(5, 3.4445, -4.7750, 2.0315, 1e-7), tag_muon_options(0.02, 0.95, 0.01, 1)
    check(P._abi.load().tag_muon_step(q, 1, C.byref(ns), C.byref(o), None, 0,
                                      torch.cuda.current_stream().cuda_stream), "tag_muon_step")
    _check(torch, w[at], m[at], w0[at], g0[at], m0[at])
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.equal(w[rest], w0[rest]) and torch.equal(m[rest], m0[rest]) and torch.equal(g, g0)


def test_many_vectors_beside_matrices(torch):
    """More plain groups than one set of launches takes, some of them long, with
    matrices that go the way of one launch and of many."""
    from paper_2302_06126_amd.optim import Muon
    for shape in ((20, 30), (90, 300)):
        params = [_arrays(torch, n, seed=n) for n in (5, 4096, 9000, 17, 4099, 1, 12288, 3, 2, 8, 6, 7, 9, 10, 11, 12, 13, 14, 4097)]
        keep = [(w.clone(), m.clone()) for w, _, m in params]
        a = torch.randn(shape, device="cuda")
        Muon([(w, g) for w, g, _ in params] + [(a, torch.randn(shape, device="cuda"))], lr=0.02, weight_decay=0.01,
             state=[m for _, _, m in params] + [torch.zeros_like(a)]).step()
        for (w, g, m), (w0, m0) in zip(params, keep):
            _check(torch, w, m, w0, g, m0)
        assert torch.isfinite(a).all()
