"""Beam search on the GPU against its plain restatement in 64 bits
(tests/_beam.py, which derives the tolerance of the totals; parents, slices and
reordered states are exact)."""
import numpy as np
import pytest

from tests import _beam as R

pytestmark = pytest.mark.gpu

WIDTHS = [(1, 1), (1, 5), (4, 4), (3, 7), (16, 16), (64, 64), (100, 3), (256, 256), (33, 256)]
SIZES = [1, 2, 3, 15, 16, 17, 60, 64, 65, 255, 256, 257, 1000, 1024, 1025, 4096, 4097, 16384, 16385, 70001]


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _say(*a):
    print(*a, flush=True)


def _type(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


class _Level:
    """A level's inputs: slices that are not allowed, beams that are not there."""

    def __init__(self, torch, seed, n, V, S, dtype="f32", done=0.0, scale=2.0, plain=False):
        rng = np.random.default_rng((2302, 61, seed))
        x = rng.normal(0, scale, (n * V, S)).astype(np.float32)
        t = (-20 * rng.random((n, V))).astype(np.float32)
        if not plain:
            x[rng.random(x.shape) < 0.2] = -np.inf
            t[:, 1:][rng.random((n, V - 1)) < 0.1] = -np.inf
        self.n, self.V, self.S, self.t = n, V, S, t
        self.x = torch.from_numpy(x).to(_type(torch, dtype))
        self.done = rng.random((n, V)) < done

    def args(self, torch):
        return self.x.cuda(), torch.from_numpy(self.t).cuda(), torch.from_numpy(self.done).cuda()

    def run(self, torch, W, x=None, **kw):
        from paper_2302_06126_amd.policy import Beam
        dx, dt, dd = self.args(torch)
        call = Beam(self.n, W, self.S, width_in=self.V, dtype=self.x.dtype)
        out = call(dx if x is None else x, dt, done=dd if self.done.any() else None, **kw)
        return [o.cpu().numpy() for o in out]

    def check(self, got, W):
        R.check(got, self.x.float().numpy().reshape(self.n, self.V, self.S), self.t, self.done, W)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", SIZES)
def test_sizes(torch, S, dtype):
    for i, (V, W) in enumerate(WIDTHS):
        if V * S > 1_500_000:
            continue
        _say(f"[beam] S={S} V={V} W={W} {dtype}")
        level = _Level(torch, S * 20 + i, 3 if V * S < 100_000 else 1, V, S, dtype, 0.2 if i % 2 else 0.0)
        level.check(level.run(torch, W), W)


@pytest.mark.parametrize("n,V,W,S", [(700, 4, 4, 60), (2000, 1, 2, 5), (300, 16, 16, 256), (17, 2, 256, 900),
                                     (317, 37, 37, 12), (9, 5, 200, 100), (9, 4, 200, 60), (6, 10, 256, 100),
                                     (70, 1, 33, 256), (70, 1, 64, 40), (1, 256, 256, 9000), (3, 200, 200, 4099)])
def test_many_searches(torch, n, V, W, S):
    _say(f"[beam] n={n} V={V} W={W} S={S}")
    level = _Level(torch, n, n, V, S, done=0.1)
    level.check(level.run(torch, W), W)


@pytest.mark.parametrize("S", [1, 7, 300, 5000, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_scores_go_by_beam_and_slice(torch, S, dtype):
    """All candidates the same; then a few better ones behind them."""
    _say(f"[beam] ties S={S} {dtype}")
    for V, W in ((1, 6), (5, 200), (64, 64)):
        level = _Level(torch, S, 2, V, S, dtype, plain=True)
        level.x.zero_()
        level.t[:] = -1.5
        level.check(level.run(torch, W), W)
        level.x[:, -1] = 1.0
        level.x[V // 2, :] = 1.0
        level.check(level.run(torch, W), W)


@pytest.mark.parametrize("V,W,S", [(256, 256, 20000), (200, 200, 4099)])
def test_equal_scores_of_long_rows(torch, V, W, S):
    """More groups of columns at the bar than are listed."""
    level = _Level(torch, S, 1, V, S, plain=True)
    level.x.zero_()
    level.t[:] = -1.5
    level.check(level.run(torch, W), W)
    level.t[:] = -np.linspace(1, 2, V).astype(np.float32)
    level.check(level.run(torch, W), W)


@pytest.mark.parametrize("V,W,S", [(200, 200, 4099), (256, 256, 17000), (64, 64, 70001), (64, 64, 256)])
def test_one_beam_of_many(torch, V, W, S):
    """The first level of a wide search, and one with the other beams finished."""
    level = _Level(torch, S, 2, V, S)
    keep = level.t[:, 3].copy()
    level.t[:] = -np.inf
    level.t[:, 3] = np.where(np.isfinite(keep), keep, -1.0)
    level.check(level.run(torch, W), W)
    level.t[0, :] = -np.arange(V, dtype=np.float32) - 40
    level.t[0, 3] = -1.0
    level.done[0, :] = True
    level.done[0, 3] = False
    level.check(level.run(torch, W), W)


@pytest.mark.parametrize("S", [40, 3000, 40000])
def test_sorted_and_clustered_scores(torch, S):
    """The best next to one another, in either order, and copies of one beam."""
    for order in (1, -1):
        for V, W in ((1, 256), (6, 40)):
            _say(f"[beam] sorted S={S} V={V} W={W} {order}")
            level = _Level(torch, S + V, 2, V, S, plain=True)
            level.x = level.x.sort(dim=1, descending=order < 0).values
            level.check(level.run(torch, W), W)
    level = _Level(torch, S, 2, 6, S, plain=True)
    level.x[:] = level.x[:1]
    level.t[:] = -3.0
    level.check(level.run(torch, 30), 30)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", [60, 300, 5000, 30000])
def test_beams_without_candidates(torch, S, dtype):
    _say(f"[beam] nothing left S={S} {dtype}")
    level = _Level(torch, S, 3, 12, S, dtype, plain=True)
    x, t = level.x, level.t
    x[0, S // 2] = float("nan")
    x[1, S - 1] = float("inf")
    x[2] = -float("inf")
    x[3, 1:] = -float("inf")                 # one slice of probability one
    x[4, 0] = torch.finfo(torch.float32).min   # (-inf in bf16)
    x[5] = torch.finfo(x.dtype).min          # every score the lowest of the type
    x[6, :] = -float("inf")
    x[6, S // 3] = torch.finfo(x.dtype).max
    t[0, 7], t[0, 8], t[0, 9] = -np.inf, np.nan, np.inf
    t[1] = -np.inf                           # a search without a beam
    level.done[0, 10] = True
    x[10, 5] = float("nan")                  # (not looked at)
    level.done[0, 8] = True                  # finished, without a total
    t[2, :] = -np.inf
    t[2, 11] = -7.25                         # the first level
    got = level.run(torch, 24)
    level.check(got, 24)
    assert (got[1][1] == -1).all() and (got[2][1] == -1).all() and np.isneginf(got[0][1]).all()
    assert set(got[1][2]) <= {11}
    assert not set(got[1][0]) & {0, 1, 2, 7, 8, 9}


def test_fewer_candidates_than_beams(torch):
    for V, S, W in ((1, 3, 8), (2, 1, 256), (5, 4, 21)):
        level = _Level(torch, V, 4, V, S, plain=True)
        got = level.run(torch, W)
        level.check(got, W)
        assert (got[1][:, V * S:] == -1).all()


def test_all_finished(torch):
    level = _Level(torch, 3, 5, 9, 50, plain=True)
    level.done[:] = True
    level.x[:] = float("nan")
    got = level.run(torch, 6)
    level.check(got, 6)
    assert (got[2] == -1).all() and np.array_equal(got[0], -np.sort(-level.t, axis=1)[:, :6])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", [37, 256, 1500, 20001])
def test_rows_anywhere(torch, S, dtype):
    """Rows of a wider tensor that start at odd elements: the same bits."""
    level = _Level(torch, S, 2, 9, S, dtype)
    base = level.run(torch, 20)
    wide = torch.full((18, S + 13), 7.0, dtype=level.x.dtype, device="cuda")
    for at in (0, 1, 2, 3, 8):
        wide[:, at:at + S] = level.x.cuda()
        got = level.run(torch, 20, x=wide[:, at:at + S])
        assert all(np.array_equal(a, b) for a, b in zip(base, got))


def test_rows_far_apart(torch):
    """Offsets beyond 2^32 bytes."""
    from paper_2302_06126_amd.policy import Beam
    S, stride = 300, (1 << 30) + 1
    level = _Level(torch, 5, 1, 5, S, "bf16")
    far = torch.empty(4 * stride + S, dtype=torch.bfloat16, device="cuda").as_strided((5, S), (stride, 1))
    far.copy_(level.x)
    got = [o.cpu().numpy() for o in Beam(1, 7, S, width_in=5, dtype=torch.bfloat16)(far, torch.from_numpy(level.t).cuda())]
    level.check(got, 7)


def test_levels_follow_one_another(torch):
    """total goes from one call into the next as it is; from the start that one object gives, and from one beam."""
    from paper_2302_06126_amd.policy import Beam
    n, W, S = 3, 8, 40
    call, first = Beam(n, W, S), Beam(n, W, S, width_in=1)
    x = _Level(torch, 1, n, W, S, plain=True).x.cuda()
    x.view(n, W, S)[:] = x.view(n, W, S)[:, :1]
    a = [o.clone() for o in call(x, call.start())]
    b = first(x.view(n, W, S)[:, 0], torch.zeros(n, 1, device="cuda"))
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])
    t = a[0]
    for i in range(4):
        level = _Level(torch, 70 + i, n, W, S)
        level.t = t.cpu().numpy()
        out = call(level.x.cuda(), call.total if i else t)
        level.check([o.cpu().numpy() for o in out], W)
        t = out[0]


def test_constrained_scores_feed_the_selection(torch):
    from paper_2302_06126_amd.policy import Beam, Constrain
    level = _Level(torch, 9, 2, 6, 200, plain=True)
    allow = np.random.default_rng(1).integers(0, 1 << 32, (12, 7), dtype=np.uint32)
    allow[3] = 0
    con = Constrain(12, 200, want_prior=False, want_scores=True)
    y = con(level.x.cuda(), allow=torch.from_numpy(allow.view(np.int32)).cuda())[3]
    got = Beam(2, 15, 200, width_in=6)(y, torch.from_numpy(level.t).cuda())
    level.x = y.cpu()
    level.check([o.cpu().numpy() for o in got], 15)
    assert not (got[1].cpu().numpy()[0] == 3).any()


@pytest.mark.parametrize("n,V,W,S", [(2, 16, 16, 60), (2, 64, 64, 3000), (1, 8, 8, 70001)])
def test_streams_and_graphs(torch, n, V, W, S):
    """Another stream; captured once, replayed with other inputs in the same
    buffers and eager calls between."""
    from paper_2302_06126_amd.policy import Beam
    levels = [_Level(torch, 90 + i, n, V, S, done=0.1) for i in range(4)]
    want = []
    for l in levels:
        got = l.run(torch, W)
        l.check(got, W)
        want.append(got)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call = Beam(n, W, S, width_in=V)
        bufs = [torch.empty_like(t) for t in levels[0].args(torch)]
    side.wait_stream(torch.cuda.current_stream())
    def fill(l):
        for b, t in zip(bufs, l.args(torch)):
            b.copy_(t)
    fill(levels[0])
    side.wait_stream(torch.cuda.current_stream())
    call(bufs[0], bufs[1], done=bufs[2], stream=side)
    side.synchronize()
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip((call.total, call.parent, call.slice), want[0]))
    other = Beam(n, W, S, width_in=V)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(bufs[0], bufs[1], done=bufs[2])
    for i in (1, 2, 3, 1, 0):
        fill(levels[i])
        graph.replay()
        eager = [o.cpu().numpy() for o in other(*levels[(i + 1) % 4].args(torch)[:2], done=levels[(i + 1) % 4].args(torch)[2])]
        torch.cuda.synchronize()
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip((call.total, call.parent, call.slice), want[i]))
        assert all(np.array_equal(a, b) for a, b in zip(eager, want[(i + 1) % 4]))


def test_calls_repeat_to_the_bit(torch):
    from paper_2302_06126_amd.policy import Beam
    level = _Level(torch, 2, 40, 16, 500, done=0.1)
    x, t, d = level.args(torch)
    call = Beam(40, 16, 500)
    first = [o.clone() for o in call(x, t, done=d)]
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(first, call(x, t, done=d)))


def test_refusals_of_tensors(torch):
    from paper_2302_06126_amd.policy import Beam
    call = Beam(2, 4, 30)
    x, t = torch.zeros(8, 30, device="cuda"), torch.zeros(2, 4, device="cuda")
    for bad in (dict(scores=x[:, :29]), dict(scores=x.to(torch.bfloat16)), dict(scores=x.cpu()), dict(total=t[:, :3]),
                dict(total=t.double()), dict(total=torch.zeros(4, 2, device="cuda").t()), dict(done=torch.zeros(2, 4, device="cuda")),
                dict(done=torch.zeros(2, 4, dtype=torch.bool)), dict(scores=torch.zeros(30, 8, device="cuda").t())):
        with pytest.raises(ValueError):
            call(**{"scores": x, "total": t, **bad})
    from paper_2302_06126_amd import TagError
    with pytest.raises(TagError):
        Beam(1, 300, 10)
    with pytest.raises(TagError):   # an output as an input of the wrong place
        call(x, call.parent.view(torch.float32))


# -------------------------------------------------------------------- reorder
def _parents(rng, n, V, W):
    p = rng.integers(0, V, (n, W)).astype(np.int32)
    p[rng.random((n, W)) < 0.15] = -1
    p.flat[0] = V
    if p.size > 3:
        p.flat[1], p.flat[2] = np.iinfo(np.int32).min, np.iinfo(np.int32).max
    return p


def _bytes(t):
    return t.contiguous().view(-1).view(t.dtype).cpu()


@pytest.mark.parametrize("n,V,W", [(1, 1, 1), (1, 4, 4), (3, 16, 16), (2, 17, 17), (1, 64, 64), (2, 200, 200), (1, 256, 256),
                                   (5, 3, 9), (2, 256, 31)])
@pytest.mark.parametrize("place", [True, False])
def test_reorder_sizes(torch, n, V, W, place):
    from paper_2302_06126_amd.policy import Reorder
    if place and V != W:
        pytest.skip("in place the width stays")
    rng = np.random.default_rng((n, V, W))
    parent = _parents(rng, n, V, W)
    for row in (1, 2, 15, 16, 17, 31, 33, 255, 256, 257, 4096, 4099, 66000):
        _say(f"[reorder] n={n} V={V} W={W} row={row} in place: {place}")
        old = rng.integers(0, 256, (n, V, row)).astype(np.uint8)
        was = old if place else rng.integers(0, 256, (n, W, row)).astype(np.uint8)
        x, y = torch.from_numpy(old).cuda(), torch.from_numpy(was).cuda()
        call = Reorder([x], n, W, width_in=V, out=None if place else [y])
        out = call(torch.from_numpy(parent).cuda())[0].cpu().numpy()
        assert np.array_equal(out, R.reorder(old, was, parent, V)), row
        if not place:
            assert np.array_equal(x.cpu().numpy(), old)


def test_reorder_many_states_at_once(torch):
    """Types and shapes of every kind, more arrays than a launch takes, parts of
    wider rows side by side, misaligned starts; guards around them stay."""
    from paper_2302_06126_amd.policy import Reorder
    n, W = 3, 10
    rng = np.random.default_rng(8)
    parent = _parents(rng, n, W, W)
    wide = torch.from_numpy(rng.integers(0, 256, (n * W, 500)).astype(np.uint8)).cuda()
    states = [wide[:, 3:40], wide[:, 40:41], wide[:, 41:400], wide[:, 403:480]]
    states += [torch.randn(n * W, 7, 5, device="cuda"), torch.randn(n, W, 33, device="cuda").to(torch.bfloat16),
               torch.randint(0, 9, (n * W,), device="cuda"), torch.randn(n, W, device="cuda").double(),
               torch.rand(n * W, 3, device="cuda") < 0.5, torch.randn(n * W, 0, device="cuda"),
               torch.randn(n, 2 * W, 6, device="cuda")[:, :W]]
    states += [torch.randn(n * W, 11 + i, device="cuda") for i in range(22)]
    old = [s.clone() for s in states]
    before = wide.clone()
    call = Reorder(states, n, W)
    call(torch.from_numpy(parent).cuda())
    for s, o in zip(states, old):
        lead = (n, W) + tuple(s.shape[1:] if s.shape[0] == n * W else s.shape[2:])
        raw = lambda t: t.reshape(lead).float().cpu().numpy() if t.dtype == torch.bfloat16 else t.reshape(lead).cpu().numpy()
        assert np.array_equal(raw(s), R.reorder(raw(o), raw(o), parent, W)), s.shape
    for lo, hi in ((0, 3), (400, 403), (480, 500)):
        assert torch.equal(wide[:, lo:hi], before[:, lo:hi])


def test_reorder_repeated_and_captured(torch):
    from paper_2302_06126_amd.policy import Reorder
    n, W = 2, 12
    rng = np.random.default_rng(3)
    x = torch.randn(n * W, 1000, device="cuda")
    p = torch.zeros(n, W, dtype=torch.int32, device="cuda")
    call = Reorder([x], n, W)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(p)
    now = x.cpu().numpy().reshape(n, W, -1)
    for i in range(6):
        parent = np.stack([rng.permutation(W) for _ in range(n)]).astype(np.int32) if i % 2 else _parents(rng, n, W, W)
        p.copy_(torch.from_numpy(parent))
        graph.replay() if i % 3 else call(p)
        now = R.reorder(now, now, parent, W)
        assert np.array_equal(x.cpu().numpy().reshape(n, W, -1), now)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(p, stream=side)
    side.synchronize()
    assert np.array_equal(x.cpu().numpy().reshape(n, W, -1), R.reorder(now, now, parent, W))


def test_reorder_rows_far_apart(torch):
    """Offsets beyond 2^32 bytes."""
    from paper_2302_06126_amd.policy import Reorder
    stride, row = (1 << 31) + 5, 1001
    far = torch.empty(3 * stride + row, dtype=torch.uint8, device="cuda").as_strided((4, row), (stride, 1))
    old = torch.randint(0, 256, (4, row), dtype=torch.uint8)
    far.copy_(old)
    parent = np.array([[3, 3, 0, 1]], np.int32)
    Reorder([far], 1, 4)(torch.from_numpy(parent).cuda())
    assert np.array_equal(far.cpu().numpy(), old.numpy()[parent[0]])


def test_reorder_refuses_tensors(torch):
    from paper_2302_06126_amd import TagError
    from paper_2302_06126_amd.policy import Reorder
    x = torch.zeros(8, 30, device="cuda")
    for states, kw in (([x.t()], {}), ([x[:, ::2]], {}), ([x], dict(out=[x.double()])), ([x], dict(out=[])),
                       ([x], dict(width_in=3)), ([x], dict(out=[torch.zeros(8, 31, device="cuda")])), ([x.cpu()], {})):
        with pytest.raises(ValueError):
            Reorder(states, 2, 4, **kw)
    call = Reorder([x], 2, 4)
    for p in (torch.zeros(2, 4, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda"),
              torch.zeros(2, 4, dtype=torch.int32)):
        with pytest.raises(ValueError):
            call(p)
    with pytest.raises(TagError):   # the same states twice
        Reorder([x, x], 2, 4)(torch.zeros(2, 4, dtype=torch.int32, device="cuda"))
    with pytest.raises(TagError):   # parents among the states
        p = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
        Reorder([p.view(8, 1)], 2, 4)(p)
