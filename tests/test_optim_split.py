"""The bound that GPU results of the Newton-Schulz products are held to
(tests/_split.py): the iteration with the kernels' roundings keeps a quarter of
it, one that loses a part of its operands does not keep it."""
import numpy as np
import pytest

from tests import _optim as R
from tests import _split as S


def gradient(seed, *shape):
    """A few strong directions over noise."""
    rng = np.random.default_rng((2302, 9, seed) + shape)
    r = max(1, min(shape) // 8)
    strong = rng.normal(0, 1, (shape[0], r)) @ rng.normal(0, 1, (r, shape[1]))
    return (1e-3 * (3 * strong / np.sqrt(r) + rng.normal(0, 1, shape))).astype(np.float32)


def _error(g, keep=(0, 1, 2)):
    want = R.newton_schulz(g)[0]
    return np.linalg.norm(S.iterate(g, keep=keep) - want) / np.linalg.norm(want)


MATRICES = {f"{s[0]}x{s[1]}": gradient(1, *s) for s in [(3, 5), (31, 33), (64, 300), (128, 256), (129, 700), (200, 200)]}
MATRICES["normal"] = np.random.default_rng(5).normal(0, 1, (150, 900)).astype(np.float32)
MATRICES["equal"] = np.full((90, 300), 0.37, np.float32)
MATRICES["repeated"] = np.repeat(gradient(2, 1, 900), 8, axis=0)
MATRICES["orthogonal"] = np.linalg.qr(np.random.default_rng(6).normal(0, 1, (150, 150)))[0].astype(np.float32)


@pytest.mark.parametrize("name", MATRICES)
def test_the_split_products_keep_the_bound(name):
    assert _error(MATRICES[name]) <= S.BOUND / 4


@pytest.mark.parametrize("keep", [(1, 2), (0, 2), (2,)])
@pytest.mark.parametrize("name", MATRICES)
def test_products_without_a_part_do_not(name, keep):
    assert _error(MATRICES[name], keep) > 8 * S.BOUND


def test_long_iterations_and_the_transpose():
    g = gradient(1, 64, 300)
    want = R.newton_schulz(g, 32)[0]
    assert np.linalg.norm(S.iterate(g, 32) - want) <= S.BOUND * np.linalg.norm(want)
    assert np.array_equal(S.iterate(g.T.copy()), S.iterate(g).T)
