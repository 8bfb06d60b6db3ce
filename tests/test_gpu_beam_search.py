"""The beam search of the search service, and a round of what stands around it:
strategies from the beam, a training step on them, clipped gradients, the
optimiser step, and the beam again.

Totals are sums of log priors of up to K levels; the priors that the service's
other path gives (the decision head's softmax in fp32) differ from the scores'
exact softmax by a few hundred half steps of fp32 each, so both agree to
K 512 2^-24 and the rounding of the totals, K 2^-24 of their magnitude."""
import numpy as np
import pytest

import synth
from oracle import search as OS
from tests import _beam as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _service(name, B, model="analytic"):
    import paper_2302_06126_amd as P0
    import paper_2302_06126_amd.search as PS
    wl = synth.WORKLOADS[name]
    sp = synth.make_search_problem(name)
    w = synth.make_weights(wl.f, wl.heads, wl.layers, wl.f_op, wl.f, bias_scale=0.5)
    gnn = P0.Model(w, f=wl.f, heads=wl.heads, layers=wl.layers, f_op=wl.f_op, dtype=wl.dtype)
    prob = PS.SearchProblem(sp, f_op=wl.f_op, model=model)
    return OS.Problem(sp, model=model), sp, gnn, prob, PS.SearchService(prob, sp, gnn, B)


def _tol(K, total):
    return K * 2.0 ** -24 * (512 + np.abs(total).max())


@pytest.mark.parametrize("name,B,depth,model", [("tiny", 8, None, "analytic"), ("tiny", 1, None, "analytic"),
                                                ("tiny", 100, 2, "simulator"), ("cnn", 16, 6, "analytic")])
def test_beam_against_the_service_s_priors(torch, name, B, depth, model):
    print(f"[beam search] {name} B={B} {model}", flush=True)
    P, sp, gnn, prob, svc = _service(name, B, model)
    paths, total, rewards = svc.beam(depth)
    K = P.K if depth is None else depth
    assert paths.shape == (len(total), K) and len(total) == min(B, P.S ** K) and np.all(np.diff(total) <= 0)
    assert len({tuple(p) for p in paths}) == len(paths)
    T_base = OS.feedback(P, OS.full_strategy(P, []))["T"]
    for p, r in zip(paths, rewards):
        assert r == pytest.approx(OS.reward(P, list(p), T_base), rel=1e-12)
    # the same search on the priors that evaluate gives
    now, sums = np.zeros((B, P.K), np.int32), np.full((1, B), -np.inf)
    sums[0, 0] = 0.0
    given = np.zeros(len(total))            # log priors along the paths that the beam found
    full = np.zeros((B, P.K), np.int32)
    full[:len(paths), :K] = paths
    for d in range(K):
        _, prior = svc.evaluate(np.full(B, d, np.int32), now)
        with np.errstate(divide="ignore"):
            x = np.log(prior.astype(np.float64))[None]
        sums, parent, choice, _ = R.select(x, sums, np.zeros((1, B), bool), B)
        now = np.where((parent[0] >= 0)[:, None], now[np.maximum(parent[0], 0)], now)
        now[:, d] = np.maximum(choice[0], 0)
        _, prior = svc.evaluate(np.full(B, d, np.int32), full)
        given += np.log(prior[np.arange(len(paths)), paths[:, d]].astype(np.float64))
    tol = _tol(K, total)
    assert np.abs(given - total).max() <= tol
    assert np.abs(sums[0, :len(total)] - total).max() <= 2 * tol
    clear = np.ones(len(total), bool)       # further than that from their neighbours: the same paths in the same places
    gaps = np.diff(sums[0, :len(total) + 1])
    clear[:len(gaps)] &= np.abs(gaps[:len(total)]) > 4 * tol
    clear[1:] &= clear[:-1]
    assert np.array_equal(now[:len(total), :K][clear], paths[clear])
    # again, and on another stream
    again = svc.beam(depth)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = svc.beam(depth, stream=side)
    for got in (again, other):
        assert all(np.array_equal(a, b) for a, b in zip(got, (paths, total, rewards)))
    svc.close()
    prob.close()


def test_beam_refuses(torch):
    _, _, _, prob, svc = _service("tiny", 2)
    for bad in (0, -1, prob.n_groups + 1):
        with pytest.raises(ValueError):
            svc.beam(bad)
    svc.close()
    prob.close()


def test_a_round_of_search_and_training(torch):
    """Strategies by the beam; the slices of the best as targets of every level's state; gradients clipped by their norm;
    the optimiser step; the beam with the new weights."""
    from paper_2302_06126_amd.optim import Clip, Muon
    from paper_2302_06126_amd.train import Trainer
    P, sp, gnn, prob, svc = _service("tiny", 8)
    B, K = 8, P.K
    levels = np.minimum(np.arange(B), K - 1).astype(np.int32)
    for turn in range(2):
        paths, total, rewards = svc.beam()
        best = paths[int(np.argmax(rewards))]
        states = np.tile(best, (B, 1)).astype(np.int32)
        svc.evaluate(levels, states)                      # (the features of these states)
        order, rep = prob.order()
        tr = Trainer(svc.graph, gnn, B, sp.masks, sp.options, np.arange(B), np.zeros(B), rep[order[levels]])
        tr.set_targets(np.eye(prob.n_slices, dtype=np.float32)[best[levels]])
        loss = tr.step(svc.feats).item()
        assert np.isfinite(loss) and loss > 0
        want = float(np.sqrt(sum((g.double() ** 2).sum().item() for g in tr.grads.values())))
        kept = {k: g.clone() for k, g in tr.grads.items()}
        weights = {k: gnn.t[k].clone() for k in tr.grads}
        muon = Muon.of(tr, max_norm=0.5 * want, lr=0.02)
        muon.step()
        assert abs(muon.norm.item() - want) <= 2.0 ** -24 * want * (1 + 1e-6)
        assert all(torch.equal(kept[k], g) for k, g in tr.grads.items())
        after = {k: gnn.t[k].clone() for k in tr.grads}
        assert all(torch.isfinite(v).all() for v in after.values())
        assert any(not torch.equal(after[k], weights[k]) for k in after)
        # the same from gradients clipped in place
        for k in weights:
            gnn.t[k].copy_(weights[k])
        clip = Clip.of(tr, 0.5 * want)
        assert torch.equal(clip(), muon.norm)
        clipped = float(np.sqrt(sum((g.double() ** 2).sum().item() for g in tr.grads.values())))
        assert abs(clipped - 0.5 * want) <= 2.0 ** -22 * want
        Muon.of(tr, lr=0.02).step()
        assert all(torch.equal(gnn.t[k], after[k]) for k in after)
    paths, total, rewards = svc.beam()
    assert np.isfinite(total).all() and np.isfinite(rewards).all()
    svc.close()
    prob.close()
