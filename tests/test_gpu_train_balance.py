"""The training step with the balance loss, and steps with the orthogonalised
update.  The balance loss's gradient b with respect to the scores sums to zero
over each query, so the step's gradients are those of the cross entropy against
the targets t - Q b: the reference training step (oracle/train.py, float64) with
such targets, b from the 64-bit restatement of the loss on the scores of the
same forward pass.  Tolerances as for the training step itself."""
import ctypes as C

import numpy as np
import pytest

import paper_2302_06126_amd as P
import synth
from oracle import train as OT
from tests import _policy as R
from tests.test_gpu_train import TrainCase, _compare

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _trainer(torch, case, balance):
    from paper_2302_06126_amd.train import Trainer
    graph, model, _, feats = case.trainer(torch)
    tr = Trainer(graph, model, case.R, case.masks, case.opts, case.q_rep, case.q_graph, case.q_op, balance=balance)
    tr.set_targets(case.target)
    return graph, model, tr, feats


def _scores(case, graph, model):
    E_op, E_dev = P.forward(graph, model, *case._keep)
    return P.scores(graph, model, E_op, E_dev, case.masks, case.opts, case.q_rep, case.q_graph, case.q_op)


@pytest.mark.parametrize("invalid", [0, 2])
@pytest.mark.parametrize("S,Q_per,coef", [(20, 3, 0.5), (300, 2, 5.0)])
def test_gradients_and_loss(torch, S, Q_per, coef, invalid):
    print(f"[train balance] S={S} Q_per={Q_per} invalid={invalid}", flush=True)
    topo = synth.random_topology(61, 30, 6, 70)
    case = TrainCase([topo], 4, 64, 4, 2, S, Q_per, seed=S + invalid, invalid=invalid)
    graph, model, tr, feats = _trainer(torch, case, coef)
    loss = float(tr.step(feats).item())
    x = _scores(case, graph, model).double().cpu().numpy()
    if invalid:
        assert np.isneginf(x[-invalid:]).all()
    bal, b, count, load, h = R.balance(x, case.masks, topo.n_dev, coef)
    assert np.array_equal(tr.count.cpu().numpy(), count) and count.sum() == case.n_valid
    assert np.abs(tr.load.cpu().numpy() - load).max() <= 2.0 ** -23
    assert abs(tr.balance_loss.item() - bal) <= 1e-5 * bal
    # the cross entropy's own loss, and the gradients of both
    ref_loss, _ = case.reference()
    assert abs(loss - (ref_loss + bal)) <= 2e-5 * (ref_loss + bal)
    Q = len(case.q_op)
    k = 0
    for it in case.items:   # (items are in the order of the queries)
        n = len(it["query_op"])
        it["target"] = np.asarray(it["target"], np.float64) - Q * b[k:k + n]
        k += n
    _, ref_g = case.reference()
    _compare(tr, ref_loss + bal, ref_loss + bal, ref_g, case.w)
    # the same bits again, and no other effect than on the step's outputs
    first = {q: v.clone() for q, v in tr.grads.items()}
    tr.balance_ws.fill_(255)
    tr.ws.fill_(255)
    tr.step(feats)
    assert all(torch.equal(first[q], tr.grads[q]) for q in first)
    graph.close()


def test_a_coefficient_of_nothing_is_the_plain_step(torch):
    topo = synth.random_topology(62, 25, 4, 50)
    case = TrainCase([topo], 2, 64, 4, 1, 30, 2, seed=9)
    graph, model, plain, feats = case.trainer(torch)
    a = plain.step(feats).clone()
    from paper_2302_06126_amd.train import Trainer
    tr = Trainer(graph, model, case.R, case.masks, case.opts, case.q_rep, case.q_graph, case.q_op, balance=1e-30)
    tr.set_targets(case.target)
    b = tr.step(feats)
    assert torch.equal(a, b) and tr.balance_loss.item() < 1e-29
    for k in plain.grads:
        assert torch.equal(plain.grads[k], tr.grads[k]), k
    graph.close()


def test_refusals(torch):
    from paper_2302_06126_amd._abi import tag_train_balance
    from paper_2302_06126_amd.train import Trainer
    topos = [synth.random_topology(63 + i, 12, 3, 20) for i in range(2)]
    two = TrainCase(topos, 1, 64, 4, 1, 8, 1, seed=3)
    graph, model, tr, feats = _trainer(torch, two, 0.1)
    with pytest.raises(P.TagError) as e:
        tr.step(feats)
    assert e.value.status == P._abi.TAG_ESHAPE
    graph.close()
    one = TrainCase(topos[:1], 1, 64, 4, 1, 8, 1, seed=3)
    graph, model, tr, feats = _trainer(torch, one, 0.1)
    for kw in (dict(coef=-1.0), dict(coef=float("nan")), dict(loss=None), dict(count=None), dict(load=None),
               dict(workspace=None), dict(ws_bytes=16), dict(loss=tr.balance.loss + 2), dict(load=tr.balance.load + 1)):
        keep, tr.balance = tr.balance, tag_train_balance.from_buffer_copy(tr.balance)
        for k, v in kw.items():
            setattr(tr.balance, k, v)
        with pytest.raises(P.TagError):
            tr.step(feats)
        tr.balance = keep
    lib = P._abi.load()
    b = C.c_size_t(0)
    assert lib.tag_train_balance_workspace(20000, 3, C.byref(b)) == P._abi.TAG_ESHAPE
    assert lib.tag_train_balance_workspace(10, 3, None) == P._abi.TAG_EINVAL
    tr.step(feats)
    graph.close()


def test_balanced_steps_with_the_orthogonalised_update(torch):
    """A few whole training steps: forward, both losses, gradients, update; captured
    and replayed they give the same parameters."""
    from paper_2302_06126_amd.optim import Muon
    topo = synth.random_topology(64, 40, 5, 90)

    def make():
        case = TrainCase([topo], 3, 64, 4, 2, 40, 2, seed=11)
        graph, model, tr, feats = _trainer(torch, case, 0.05)
        return case, graph, model, tr, feats, Muon.of(tr, lr=0.01, weight_decay=0.01)

    case, graph, model, tr, feats, opt = make()
    for _ in range(4):
        tr.step(feats)
        opt.step()
    assert all(torch.isfinite(t).all() for t in model.t.values()) and torch.isfinite(tr.loss).all()
    case2, graph2, model2, tr2, feats2, opt2 = make()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        tr2.step(feats2)
        opt2.step()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        tr2.step(feats2)
        opt2.step()
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
    for k in model.t:
        assert torch.equal(model.t[k], model2.t[k]), k
    graph.close()
    graph2.close()
