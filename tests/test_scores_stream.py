"""Decide.scores on a given stream, without a GPU: the tensor that the first call
makes is memory of the graph's device, so it is that device's stream that the
given one waits for, whichever device is current."""
from types import SimpleNamespace

import paper_2302_06126_amd as P


class _Stream:
    cuda_stream = 77

    def __init__(self):
        self.waited = []

    def wait_stream(self, other):
        self.waited.append(other)


def test_the_stream_waits_for_the_graphs_device(monkeypatch):
    made = []

    def empty(shape, dtype=None, device=None):
        made.append((tuple(shape), device))
        return SimpleNamespace(data_ptr=lambda: 4096)

    cuda = SimpleNamespace(current_stream=lambda device=None: SimpleNamespace(device=device, cuda_stream=5))
    monkeypatch.setattr(P, "_torch", lambda: SimpleNamespace(empty=empty, cuda=cuda, float32="f32"))
    monkeypatch.setattr(P, "_ptr", lambda t: None)
    calls = []
    monkeypatch.setattr(P, "tag_gnn_scores", lambda *a: calls.append(a[-1]) or 0)
    d = object.__new__(P.Decide)
    d.graph, d.model = SimpleNamespace(handle=1, device="cuda:1"), SimpleNamespace(dims=None, weights=None)
    d.R, d.S, d.Q, d.slices, d.q, d.ws, d.ws_bytes, d.score = 1, 5, 3, None, [None] * 3, None, 16, None
    s = _Stream()
    first = d.scores(None, None, stream=s)
    assert made == [((3, 5), "cuda:1")] and [w.device for w in s.waited] == ["cuda:1"] and calls == [77]
    assert d.scores(None, None, stream=s) is first and len(made) == 1 and len(s.waited) == 1
    d.score = None
    d.scores(None, None)   # (without a stream there is nothing to wait for)
    assert len(s.waited) == 1
