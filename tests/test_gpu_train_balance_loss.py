"""The balance part of a step's loss and their sum are two places: with one for
both, the sum would be twice the cross entropy."""
import pytest

import paper_2302_06126_amd as P
import synth
from tests.test_gpu_train import TrainCase
from tests.test_gpu_train_balance import _trainer, torch  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def test_one_place_for_both_losses_is_refused(torch):   # noqa: F811
    case = TrainCase([synth.random_topology(65, 20, 4, 40)], 2, 64, 4, 1, 20, 2, seed=5)
    graph, model, tr, feats = _trainer(torch, case, 0.5)
    both = float(tr.step(feats))
    part = float(tr.balance_loss)
    assert both > part > 0
    keep = tr.balance.loss
    tr.balance.loss = tr.loss.data_ptr()
    with pytest.raises(P.TagError) as e:
        tr.step(feats)
    assert e.value.status == P._abi.TAG_EINVAL
    tr.balance.loss = keep
    assert float(tr.step(feats)) == both and float(tr.balance_loss) == part
    graph.close()
