"""Wide searches near their end, on the GPU: almost every beam is finished, so that few
of a block's threads have a candidate (a finished beam's one stands in its first
group of columns; where a row's groups are a multiple of 64, those of all rows
belong to the same few threads)."""
import numpy as np
import pytest

from tests.test_gpu_beam import _Level, _say, torch  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,S", [(256, 4096), (200, 4096), (64, 8192), (256, 4099), (100, 65536), (64, 65537)])
@pytest.mark.parametrize("left", [0, 1, 2, 3])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_all_but_a_few_finished(torch, V, S, left, dtype):   # noqa: F811
    _say(f"[beam] V={V} S={S} {left} left {dtype}")
    level = _Level(torch, V + S + left, 2, V, S, dtype)
    level.done[:] = True
    for b in range(2):
        at = np.random.default_rng(left + b).permutation(V)[:left]
        level.done[b, at] = False
        level.t[b, at] = -0.5 - np.arange(left, dtype=np.float32)
    for W in (V, 3, 256):
        got = level.run(torch, W)
        level.check(got, W)
        assert left or (got[2] == -1).all()
