"""States without elements, on the CPU: however their axes stand, a beam's part of
them is contiguous and of no bytes."""
import pytest


@pytest.mark.parametrize("shape", [(8, 0), (8, 0, 5), (8, 5, 0), (8, 5, 0, 3), (2, 4, 0), (2, 4, 5, 0), (2, 4, 5, 0, 3)])
def test_rows_of_no_bytes(shape):
    import torch
    from paper_2302_06126_amd.policy import Reorder
    call = Reorder.__new__(Reorder)
    call.n, call.device = 2, torch.device("cpu")
    row, search, beam = call._layout(torch.zeros(shape), 4)
    assert row == 0 and search >= 0 and beam >= 0
