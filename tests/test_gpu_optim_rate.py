"""A rate that a step refuses is not kept for the following ones."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("nan"), -1.0, float("inf")])
def test_a_refused_rate_leaves_the_object_as_it_was(bad):
    import torch
    from paper_2302_06126_amd import TagError
    from paper_2302_06126_amd.optim import Muon
    w, g = torch.randn(20, 30, device="cuda"), torch.randn(20, 30, device="cuda")
    v = w.clone()
    a, b = Muon([(w, g)], lr=0.1), Muon([(v, g)], lr=0.1)
    for opt in (a, b):
        opt.step(lr=0.05)
    was = a.m[0].clone()
    with pytest.raises(TagError):
        a.step(lr=bad)
    assert torch.equal(w, v) and torch.equal(a.m[0], was)
    a.step()
    b.step()
    assert torch.equal(w, v) and torch.equal(a.m[0], b.m[0])
