"""bf16 matrices of every size are orthogonalised to the accuracy of fp32 ones and
rounded once.  Rounding a value that is off by d errs by at most d more than
rounding the value itself, so with d of the 2-norm at most _split.BOUND a result's
error is at most its own rounding's and 2 d."""
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


def _matrix(kind, shape):
    rng = np.random.default_rng((2302, 12) + shape)
    if kind == "equal":
        return np.full(shape, 0.37, np.float32)
    if kind == "repeated":   # (each row eight times)
        return np.repeat(gradient(3, -(-shape[0] // 8), shape[1]), 8, axis=0)[:shape[0]]
    if kind == "orthogonal":
        return np.linalg.qr(rng.normal(0, 1, shape))[0].astype(np.float32)
    return gradient(3, *shape) if kind == "gradient" else rng.normal(0, 1, shape).astype(np.float32)


CASES = [("equal", (300, 300), 5), ("equal", (100, 2000), 5), ("repeated", (300, 900), 5), ("repeated", (8, 2000), 5),
         ("orthogonal", (300, 300), 5), ("gradient", (1, 300), 5), ("gradient", (300, 1), 5), ("gradient", (520, 2100), 5),
         ("gradient", (65, 65), 5), ("normal", (96, 96), 5), ("normal", (1024, 1024), 5), ("gradient", (100, 300), 32)]


@pytest.mark.parametrize("kind,shape,steps", CASES)
def test_errors_are_the_results_rounding(torch, kind, shape, steps):
    from paper_2302_06126_amd.optim import orthogonalise
    t = torch.from_numpy(_matrix(kind, shape)).to(torch.bfloat16)
    want = R.newton_schulz(t.double().numpy(), steps)[0]
    rounding = np.linalg.norm(torch.from_numpy(want).to(torch.bfloat16).double().numpy() - want)
    size = np.linalg.norm(want)
    # (32 steps go through singular values near one again and again: 1.8e-5 in the iteration with the kernels' roundings)
    d = S.BOUND * (4 if steps > 5 else 1) * size
    err = np.linalg.norm(orthogonalise(t.cuda(), steps=steps).double().cpu().numpy() - want)
    print(f"   {kind} {shape}: {err / size:.2e}, its rounding {rounding / size:.2e}", flush=True)
    assert err <= rounding + 2 * d


@pytest.mark.parametrize("count,shape", [(1, (65, 64)), (3, (64, 257)), (2, (300, 900)), (1, (900, 300)), (4, (1024, 1030)),
                                         (40, (130, 70))])
def test_results_are_the_rounded_fp32_ones(torch, count, shape):
    from paper_2302_06126_amd.optim import orthogonalise
    t = torch.from_numpy(np.stack([gradient(i, *shape) for i in range(count)])).to(torch.bfloat16).cuda()
    assert torch.equal(orthogonalise(t), orthogonalise(t.float()).to(torch.bfloat16))


def test_neighbours_do_not_change_the_accuracy(torch):
    """A small matrix beside a large one, and in the second set of groups."""
    from paper_2302_06126_amd.optim import Orthogonalise
    shapes = [(1, 64, 64)] * 2 + [(1, 300, 300)] + [(1, 40, 50)] * 9
    xs = [torch.from_numpy(_matrix("equal" if i < 1 else "gradient", s[1:])).to(torch.bfloat16)[None] for i, s in enumerate(shapes)]
    for x, y in zip(xs, Orthogonalise(shapes, dtype=torch.bfloat16)([x.cuda() for x in xs])):
        want = R.newton_schulz(x[0].double().numpy())[0]
        rounding = np.linalg.norm(torch.from_numpy(want).to(torch.bfloat16).double().numpy() - want)
        assert np.linalg.norm(y[0].double().cpu().numpy() - want) <= rounding + 2 * S.BOUND * np.linalg.norm(want)
