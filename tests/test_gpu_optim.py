"""Orthogonalised updates on the GPU, against the iteration in 64 bits by singular
values (tests/_optim.py, where the tolerances are derived)."""
import numpy as np
import pytest

from tests import _optim as R

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _say(*a):
    print(*a, flush=True)


def _matrix(seed, *shape, kind="gradient"):
    rng = np.random.default_rng((2302, 9, seed) + tuple(shape))
    g = rng.normal(0, 1, shape)
    if kind == "gradient":   # a few strong directions over noise
        r = max(1, min(shape[-2:]) // 8)
        strong = rng.normal(0, 1, shape[:-2] + (shape[-2], r)) @ rng.normal(0, 1, shape[:-2] + (r, shape[-1]))
        g = 1e-3 * (3 * strong / np.sqrt(r) + g)
    return g.astype(np.float32)


def _check(got, g, steps=5, coef=R.QUINTIC, eps=1e-7, bf16=False):
    want, norms = R.newton_schulz(g, steps, coef, eps)
    fro, el = R.tolerance(g.shape, norms, steps, bf16)
    err = np.asarray(got, np.float64) - want
    own = np.abs(want) * 2.0 ** -8 if bf16 else 0.0
    size = np.linalg.norm(err) - (2.0 ** -8 * np.linalg.norm(want) if bf16 else 0.0)
    _say(f"   {g.shape}: {np.linalg.norm(err):.2e} of {np.linalg.norm(want):.2e}, tolerance {fro:.2e}")
    assert size <= fro, (size, fro)
    assert np.all(np.abs(err) <= el + own), float((np.abs(err) - own).max() / el)


SHAPES = [(1, 1), (1, 2), (2, 1), (1, 300), (300, 1), (3, 5), (16, 16), (31, 33), (63, 65), (64, 64), (64, 42), (65, 64),
          (128, 256), (100, 516), (257, 130), (256, 8), (400, 400), (129, 700)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalise_shapes(torch, shape, dtype):
    from paper_2302_06126_amd.optim import orthogonalise
    _say(f"[orthogonalise] {shape} {dtype}")
    t = torch.from_numpy(_matrix(1, *shape)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    got = orthogonalise(t.cuda())
    assert got.dtype == t.dtype and got.shape == t.shape
    _check(got.float().cpu().numpy(), t.float().numpy(), bf16=dtype == "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,shape", [(1, (1024, 1024)), (3, (900, 700)), (2, (520, 2100)), (40, (70, 130))])
def test_orthogonalise_large_tiles(torch, count, shape, dtype):
    """Enough tiles of 128 x 128 to be taken, ragged ones among them."""
    from paper_2302_06126_amd.optim import orthogonalise
    _say(f"[orthogonalise] {count} of {shape} {dtype}")
    t = torch.from_numpy(_matrix(2, count, *shape)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    got = orthogonalise(t.cuda()).float().cpu().numpy()
    for i in sorted({0, count - 1}):
        _check(got[i], t[i].float().numpy(), bf16=dtype == "bf16")


@pytest.mark.parametrize("shape", [(64, 1024), (8, 2000), (256, 256), (300, 900), (700, 500)])
@pytest.mark.parametrize("kind", ["gradient", "normal"])
def test_bf16_loses_little_beside_the_results_rounding(torch, shape, kind):
    """The result is a rounding to bf16 of an iteration with the roundings of
    rounded_bf16.  It strays from that by fp32 sums (2^-17 and less of ||X||, see
    tests/_optim.py) that now and then turn an operand's rounding (2^-10 of the
    operand; one in 2^6 of them at 2^-17 over a spacing of 2^-11, so 2^-3 of the
    roundings' own effect, which is below 2^-8): 2^-11 in all.  Without the
    diagonals apart the error is 1.5 to 2.3 times the rounding's."""
    from paper_2302_06126_amd.optim import orthogonalise
    t = torch.from_numpy(_matrix(8, *shape, kind=kind)).to(torch.bfloat16)
    g = t.double().numpy()
    exact, want = R.newton_schulz(g)[0], R.rounded_bf16(g)
    rounding = np.linalg.norm(torch.from_numpy(want).to(torch.bfloat16).double().numpy() - want)
    size = np.linalg.norm(exact)
    got = orthogonalise(t.cuda()).double().cpu().numpy()
    err = np.linalg.norm(got - exact)
    _say(f"   {shape} {kind}: {err / size:.2e}, of it the result's rounding {rounding / size:.2e}, the operands' "
         f"{np.linalg.norm(want - exact) / size:.2e}")
    assert err <= rounding + np.linalg.norm(want - exact) + 2.0 ** -11 * size


@pytest.mark.parametrize("shape", [(5, 9), (64, 256), (42, 64), (200, 30)])
def test_small_bf16_matrices_are_the_rounded_fp32_ones(torch, shape):
    """Up to 64 x 256 both types take products of both parts: the same sums, rounded once at the end."""
    from paper_2302_06126_amd.optim import orthogonalise
    t = torch.from_numpy(_matrix(9, 3, *shape)).to(torch.bfloat16).cuda()
    assert torch.equal(orthogonalise(t), orthogonalise(t.float()).to(torch.bfloat16))


@pytest.mark.parametrize("steps,coef", [(1, R.QUINTIC), (2, R.QUINTIC), (3, (2.0, -1.5, 0.5)), (12, (1.5, -0.5, 0.0)),
                                        (6, (3.0, -3.2, 1.2))])
def test_orthogonalise_other_iterations(torch, steps, coef):
    from paper_2302_06126_amd.optim import orthogonalise
    g = _matrix(3, 90, 150)
    _say(f"[orthogonalise] {steps} steps of {coef}")
    _check(orthogonalise(torch.from_numpy(g).cuda(), steps=steps, coef=coef).cpu().numpy(), g, steps, coef)


def test_orthogonalise_sizes_of_values(torch):
    """Gradients whose squares leave the range of fp32, powers of two apart; zeros;
    an eps that matters; infinities and NaN in one matrix of several."""
    from paper_2302_06126_amd.optim import orthogonalise
    g = _matrix(4, 70, 90, kind="noise")
    base = orthogonalise(torch.from_numpy(g).cuda(), eps=1e-30).cpu().numpy()
    _check(base, g, eps=1e-30)
    for e in (-70, -30, 30, 100):
        scaled = np.ldexp(g, e)
        _say(f"[orthogonalise] values times 2^{e}")
        assert np.array_equal(orthogonalise(torch.from_numpy(scaled).cuda(), eps=1e-37).cpu().numpy(),
                              orthogonalise(torch.from_numpy(g).cuda(), eps=1e-37).cpu().numpy()) or e == -70
        _check(orthogonalise(torch.from_numpy(scaled).cuda(), eps=1e-37).cpu().numpy(), scaled, eps=1e-37)
    assert not orthogonalise(torch.zeros(3, 5, 7, device="cuda")).any()
    _check(orthogonalise(torch.from_numpy(g).cuda(), eps=50.0).cpu().numpy(), g, eps=50.0)
    three = np.stack([g, g, g])
    three[1, 3, 4] = np.nan
    three[2, 0, 0] = np.inf
    out = orthogonalise(torch.from_numpy(three).cuda(), eps=1e-30).cpu().numpy()
    assert np.array_equal(out[0], base) and np.isnan(out[1:]).all()


def test_orthogonalise_strides_and_in_place(torch):
    """Halves of wider rows (their matrices interleaved), transposes' shapes, results
    in place, and everything around them left as it was."""
    from paper_2302_06126_amd.optim import Orthogonalise, orthogonalise
    f = 48
    w = torch.from_numpy(_matrix(5, 4, f, 2 * f)).cuda()
    keep = w.clone()
    want = [orthogonalise(w[:, :, :f].contiguous()), orthogonalise(w[:, :, f:].contiguous())]
    call = Orthogonalise([(4, f, f), (4, f, f)])
    call([w[:, :, :f], w[:, :, f:]], out=[w[:, :, :f], w[:, :, f:]])
    assert torch.equal(w[:, :, :f], want[0]) and torch.equal(w[:, :, f:], want[1])
    wide = torch.full((6, 40, 71), 5.0, device="cuda")
    x = torch.from_numpy(_matrix(6, 6, 37, 64)).cuda()
    call = Orthogonalise([(6, 37, 64)])
    call([x], out=[wide[:, 1:38, 3:67]])
    assert torch.equal(wide[:, 1:38, 3:67], orthogonalise(x))
    wide[:, 1:38, 3:67] = 5.0
    assert (wide == 5.0).all() and not torch.equal(keep, w)
    woven = torch.zeros(30, 4, 20, device="cuda")   # row r of matrix i at [r][i]
    y = torch.from_numpy(_matrix(7, 4, 30, 20)).cuda()
    Orthogonalise([(4, 30, 20)])([y], out=[woven.permute(1, 0, 2)])
    assert torch.equal(woven.permute(1, 0, 2), orthogonalise(y))


def test_orthogonalise_many_groups(torch):
    """More groups than one set of launches takes; a group's result does not depend
    on its neighbours beyond the tile size that the whole set takes."""
    from paper_2302_06126_amd.optim import Orthogonalise
    rng = np.random.default_rng(11)
    shapes = [(int(rng.integers(1, 4)), int(rng.integers(1, 150)), int(rng.integers(1, 150))) for _ in range(37)]
    xs = [_matrix(i, *s) for i, s in enumerate(shapes)]
    out = Orthogonalise(shapes)([torch.from_numpy(x).cuda() for x in xs])
    for s, x, y in zip(shapes, xs, out):
        for i in range(s[0]):
            _check(y[i].cpu().numpy(), x[i])


def test_orthogonalise_refusals(torch):
    from paper_2302_06126_amd import TagError
    from paper_2302_06126_amd.optim import Muon, Orthogonalise, orthogonalise
    x = torch.ones(2, 8, 8, device="cuda")
    call = Orthogonalise([(2, 8, 8)])
    for bad in (x.double(), x.cpu(), x[:1], x[:, :7], x.transpose(1, 2)[:, :, :8].transpose(1, 2).transpose(1, 2)):
        with pytest.raises(ValueError):
            call([bad])
    with pytest.raises(ValueError):
        call([x, x])
    with pytest.raises(ValueError):
        orthogonalise(x.half())
    with pytest.raises(TagError):
        orthogonalise(x, steps=0)
    with pytest.raises(TagError):
        orthogonalise(x, coef=(9.0, 0.0, 0.0))
    with pytest.raises(TagError):   # one matrix written twice
        call([x], out=[x[:1].expand(2, 8, 8)])
    for params in ([], [(x, x[:1])], [(x.cpu(), x.cpu())]):
        with pytest.raises(ValueError):
            Muon(params)
    with pytest.raises(TagError):
        Muon([(x, x)]).step()
    with pytest.raises(TagError):
        Muon([(x, x + 1)], momentum=1.0).step()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 300), (5, 9), (300, 64), (70, 300)])
def test_matrices_that_are_not_finite_stay_alone(torch, shape, dtype):
    from paper_2302_06126_amd.optim import orthogonalise
    x = torch.from_numpy(_matrix(10, 4, *shape)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    clean = orthogonalise(x)
    x[1, -1, 0], x[2, 0, -1], x[3] = float("nan"), float("-inf"), 0.0
    y = orthogonalise(x)
    assert torch.equal(y[0], clean[0]) and torch.isfinite(y[0]).all()
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all() and not y[3].any()


def test_arrays_given_twice_are_refused(torch):
    from paper_2302_06126_amd.optim import Muon, Orthogonalise
    x, y, g = (torch.ones(1, 8, 8, device="cuda") for _ in range(3))
    call = Orthogonalise([(1, 8, 8), (1, 8, 8)])
    for matrices, out in (([x, y], [y, x]), ([x, y], [g, g]), ([x, x], [x, y])):
        with pytest.raises(ValueError):
            call(matrices, out=out)
    call([x, y], out=[x, g])
    with pytest.raises(ValueError):   # one weight twice, one momentum for two
        Muon([(x, g), (x, g)])
    with pytest.raises(ValueError):
        Muon([(x, g), (y, g)], state=[torch.zeros_like(x)[:]] * 2)
    Muon([(x, g), (y, g)]).step()     # (a shared gradient is only read)


# ----------------------------------------------------------------------- muon
def _muon_reference(w, g, m, lr, mu, nesterov, wd, steps):
    """steps of the update in 64 bits (w, m), gradients held."""
    w, g, m = (np.asarray(v, np.float64) for v in (w, g, m))
    for _ in range(steps):
        m = mu * m + g
        u = g + mu * m if nesterov else m
        if w.ndim == 1:
            o = u
        else:
            o = np.stack([R.newton_schulz(v)[0] for v in u.reshape((-1,) + u.shape[-2:])]).reshape(u.shape)
            o = o * np.sqrt(max(1.0, w.shape[-2] / w.shape[-1]))
        w = (1 - lr * wd) * w - lr * o
    return w, m


@pytest.mark.parametrize("nesterov,mu,wd", [(True, 0.95, 0.01), (False, 0.9, 0.0), (True, 0.0, 0.5)])
def test_muon_steps(torch, nesterov, mu, wd):
    from paper_2302_06126_amd.optim import Muon
    rng = np.random.default_rng((5, int(mu * 100)))
    shapes = [(3, 64, 128), (90, 20), (1, 33), (700,), (40, 40), (1,), (2, 130, 70)]
    ws = [rng.normal(0, 0.1, s).astype(np.float32) for s in shapes]
    gs = [_matrix(i, *s) if len(s) > 1 else rng.normal(0, 1e-3, s).astype(np.float32) for i, s in enumerate(shapes)]
    ms = [rng.normal(0, 1e-3, s).astype(np.float32) for s in shapes]
    W, G, M = ([torch.from_numpy(v).cuda() for v in vs] for vs in (ws, gs, ms))
    opt = Muon(list(zip(W, G)), lr=0.02, momentum=mu, nesterov=nesterov, weight_decay=wd, state=M)
    for _ in range(2):
        opt.step()
    opt.step(lr=0.01)
    for i, s in enumerate(shapes):
        w1, m1 = _muon_reference(ws[i], gs[i], ms[i], 0.02, mu, nesterov, wd, 2)
        w1, m1 = _muon_reference(w1, gs[i], m1, 0.01, mu, nesterov, wd, 1)
        # momentum: three roundings a step, of values below their sum
        size = np.abs(ms[i]) + 3 * np.abs(gs[i])
        assert np.all(np.abs(M[i].cpu().numpy() - m1) <= 9 * EPS32 * size), s
        # weights: the roundings of three updates and lr times the error of O
        err = np.abs(W[i].cpu().numpy() - w1)
        if len(s) == 1:
            tol = 12 * EPS32 * (np.abs(ws[i]) + 0.06 * size * 2)
        else:
            u = gs[i].reshape((-1,) + gs[i].shape[-2:])
            el = max(R.tolerance(v.shape, R.newton_schulz(v)[1])[1] for v in u)
            # (the rounding of m, 9 half steps of it, raised like the first X: by at most 4^5 of its share of the norm)
            el += 4.0 ** 5 * 9 * EPS32 * 10 / np.sqrt(min(s[-2:]) * 1.0 * max(s[-2:]))
            tol = 12 * EPS32 * (np.abs(ws[i]) + 0.1) + 0.05 * el * np.sqrt(max(1.0, s[-2] / s[-1]))
        assert np.all(err <= tol), (s, float((err / tol).max()))
        assert torch.equal(G[i].cpu(), torch.from_numpy(gs[i]))


def test_muon_without_a_rate_updates_the_momentum_alone(torch):
    from paper_2302_06126_amd.optim import Muon
    w, g = torch.randn(30, 50, device="cuda"), torch.randn(30, 50, device="cuda")
    v, h = torch.randn(9, device="cuda"), torch.randn(9, device="cuda")
    keep = [w.clone(), v.clone()]
    opt = Muon([(w, g), (v, h)], lr=0.0, momentum=0.5)
    opt.step()
    opt.step()
    assert torch.equal(w, keep[0]) and torch.equal(v, keep[1])
    assert torch.equal(opt.m[0], g * 1.5) and torch.equal(opt.m[1], h * 1.5)


def test_repeatable_on_streams_and_in_graphs(torch):
    """The same bits from every call, on a stream of its own, and from two graphs
    whose objects have their own workspaces, replayed in turn between eager calls."""
    from paper_2302_06126_amd.optim import Muon, Orthogonalise
    xs = [torch.from_numpy(_matrix(i, 2, 100, 60 + 80 * i)).cuda() for i in range(2)]
    want = [Orthogonalise([tuple(x.shape)])([x])[0] for x in xs]
    s = torch.cuda.Stream()
    calls, graphs, outs = [], [], []
    for x in xs:
        call = Orthogonalise([tuple(x.shape)])
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            call([x])
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(call([x])[0])
        calls.append(call)
        graphs.append(g)
    for i in range(3):
        for x, g, o, w in zip(xs, graphs, outs, want):
            o.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, w), i
            assert torch.equal(Orthogonalise([tuple(x.shape)])([x])[0], w)
    calls[0].ws.fill_(255)
    calls[0]([xs[0]], stream=s)
    s.synchronize()
    assert torch.equal(outs[0], want[0])
    # an optimiser step in a graph: each replay is one more step
    def make():
        w = torch.from_numpy(_matrix(21, 50, 80)).cuda()
        return w, Muon([(w, torch.from_numpy(_matrix(22, 50, 80)).cuda())], lr=0.1)
    w, opt = make()
    for _ in range(4):
        opt.step()
    w2, opt2 = make()
    with torch.cuda.stream(s):
        opt2.step()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        opt2.step()
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
    assert torch.equal(w, w2) and torch.equal(opt.m[0], opt2.m[0])


def test_muon_of_a_trainer(torch):
    """Training steps of the GNN with the orthogonalised update: the trainer's
    gradients, every parameter updated as the 64-bit update of them."""
    import paper_2302_06126_amd as P
    import synth
    from paper_2302_06126_amd.optim import Muon
    from paper_2302_06126_amd.train import PARAM_NAMES, Trainer
    f, layers, H, R_ = 64, 2, 32, 3
    topo = synth.random_topology(41, 30, 4, 60)
    rng = np.random.default_rng(17)
    weights = synth.make_weights(f, 4, layers, 42, H, bias_scale=0.3, seed_extra=2)
    graph = P.Graph([topo])
    model = P.Model(weights, f=f, heads=4, layers=layers, f_op=42, dec_hidden=H)
    masks, opts = synth.make_slices("cnn", 4, 20)
    q_op = rng.integers(0, 30, R_).astype(np.int32)
    tr = Trainer(graph, model, R_, masks, opts, np.arange(R_), np.zeros(R_), q_op)
    t = rng.random((R_, 20)).astype(np.float32)
    tr.set_targets(t / t.sum(axis=1, keepdims=True))
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    xs = [d(rng.uniform(-1, 1, s).astype(np.float32)) for s in ((R_, 30, 42), (R_, 4, 8), (topo.e_oo,), (topo.e_dd, 2))]
    xs.append(d(rng.integers(0, 2, topo.e_od).astype(np.uint8)))
    feats = P.make_features(*xs)
    opt = Muon.of(tr, lr=0.02, weight_decay=0.1)
    assert sum(w.numel() for w, _ in opt.params) == sum(model.t[k].numel() for k in PARAM_NAMES)
    for _ in range(2):
        was = {k: model.t[k].clone() for k in PARAM_NAMES}
        moms = {k: m.clone() for k, m in zip(PARAM_NAMES, opt.m)}
        loss = tr.step(feats)
        assert torch.isfinite(loss).all()
        opt.step()
        for k, (w, g), m in zip(PARAM_NAMES, opt.params, opt.m):
            assert w.data_ptr() == model.t[k].data_ptr()
            w1, m1 = _muon_reference(was[k].view(w.shape).cpu().numpy(), g.cpu().numpy(), moms[k].cpu().numpy(), 0.02,
                                     0.95, True, 0.1, 1)
            size = moms[k].abs().cpu().numpy() + g.abs().cpu().numpy()
            assert np.all(np.abs(m.cpu().numpy() - m1) <= 3 * EPS32 * size + 1e-45), k
            err = np.abs(w.cpu().numpy() - w1)
            if w.dim() == 1:
                tol = 4 * EPS32 * (np.abs(w1) + 0.1 * size) + 1e-45
            else:
                u = (g + 0.95 * m).cpu().numpy().reshape((-1,) + tuple(w.shape[-2:]))
                el = max(R.tolerance(v.shape, R.newton_schulz(v)[1])[1] for v in u)
                el += 4.0 ** 5 * 4 * EPS32 * 10 / np.sqrt(w.shape[-2] * w.shape[-1])
                tol = 4 * EPS32 * (np.abs(w1) + 0.1) + 0.02 * el * np.sqrt(max(1.0, w.shape[-2] / w.shape[-1]))
            assert np.all(err <= tol), (k, float((err / tol).max()))
    graph.close()
