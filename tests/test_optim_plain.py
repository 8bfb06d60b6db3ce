"""Which sizes of plain groups (vectors, momentum SGD) the optimiser step takes, on
either side of the limit: 2^31 elements, counted by blocks of 4,096 of a matrix."""
import ctypes as C

import pytest

EINVAL, ESHAPE = -1, -4


@pytest.fixture(scope="module")
def abi():
    import paper_2302_06126_amd as P
    P._abi.load()
    return P._abi


def _workspace(abi, count, rows, cols, plain=1):
    g = (abi.tag_muon_group * 1)()
    g[0].count, g[0].rows, g[0].cols, g[0].plain = count, rows, cols, plain
    b = C.c_size_t(7)
    return abi.load().tag_muon_workspace(g, 1, C.byref(b)), b.value


@pytest.mark.parametrize("shape", [(1, 1, 2 ** 25), (1, 1, 2 ** 25 + 1), (1, 1, 2 ** 26), (1, 1, 2 ** 31 - 1),
                                   (2, 1, 2 ** 30), (1, 65536, 32768), (1, 2 ** 20, 2 ** 11), (1, 2 ** 31 - 1, 1),
                                   (2 ** 19, 1, 4096), (2 ** 19, 1, 1), (2 ** 18, 1, 8192)])
def test_plain_groups_up_to_the_limit(abi, shape):
    assert _workspace(abi, *shape) == (0, 0)


@pytest.mark.parametrize("shape", [(2, 1, 2 ** 31 - 1), (1, 65536, 32769), (2 ** 19, 1, 4097), (2 ** 19 + 1, 1, 1),
                                   (2 ** 31 - 1, 1, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)])
def test_plain_groups_past_the_limit(abi, shape):
    assert _workspace(abi, *shape)[0] == ESHAPE


def test_matrices_keep_their_own_limits(abi):
    for shape in [(1, 32768, 32768), (2, 32768, 32768), (2 ** 19, 64, 64), (2 ** 19, 1, 1)]:
        st, b = _workspace(abi, *shape, plain=0)
        assert st == 0 and b > 0
    for shape in [(1, 1, 32769), (3, 32768, 32768), (2 ** 19, 64, 65), (2 ** 19 + 1, 1, 1)]:
        assert _workspace(abi, *shape, plain=0)[0] == ESHAPE
    assert _workspace(abi, 0, 1, 5)[0] == EINVAL
