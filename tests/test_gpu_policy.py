"""The operators on scores on the GPU, against their plain restatements in 64
bits (tests/_policy.py).

Tolerances, in half steps of fp32 (2^-24, relative).  Constrained scores,
argmax and counts are exact: the header fixes the order of the fp32 operations.
A prior is e^(y - max) / sum: rounding y - max costs at most its magnitude in
half steps, the exponential 4 (two of a hardware step, two of its correction),
the sum as much again as its terms and log2 of their number, the reciprocal and
the product 3: fewer than 2 range + 64 with the range of y below its maximum
that is not yet zero (at most 88).  The gradient f p (h - mean) has the same
factors twice over and h, of magnitude H, rounded three times.  bf16 results are
off by half a step of theirs (2^-8 relative... 2^-9 of the value's binade) more.
"""
import ctypes as C

import numpy as np
import pytest

from tests import _policy as R

pytestmark = pytest.mark.gpu

SIZES = [1, 2, 3, 31, 32, 33, 60, 64, 65, 101, 255, 256, 257, 1000, 1024, 1025, 4095, 4096, 4097, 8191, 8192, 8193,
         12288, 16383, 16384, 16385, 20003, 70001]


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _say(*a):
    print(*a, flush=True)


def _bf16(torch, a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16)


def _words(rng, rows, S, keep=0.75):
    bits = rng.random((rows, S)) < keep
    pad = np.zeros((rows, (S + 31) // 32 * 32), bool)
    pad[:, :S] = bits
    return np.packbits(pad, axis=1, bitorder="little").view(np.uint32)


def _check_prior(got, want, y):
    """got fp32 against want in 64 bits."""
    assert np.array_equal(np.isnan(got), np.isnan(want))
    rng_ = 88.0
    ok = ~np.isnan(want)
    err = np.abs(got.astype(np.float64) - want)[ok]
    tol = (2 * rng_ + 64) * R.EPS * want[ok] + 2.0 ** -125   # (values below the normal range are flushed)
    assert np.all(err <= tol), float((err / tol).max())


class _Case:
    """Scores with everything that may stand in them, and the constraints."""

    def __init__(self, seed, Q, S, dtype, per_row=True, T=17):
        import torch
        rng = np.random.default_rng((2302, 5, seed))
        x = rng.normal(0, 3, (Q, S)).astype(np.float32)
        self.t = torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        self.rows = Q if per_row else 1
        self.allow = _words(rng, self.rows, S)
        self.bias = rng.normal(0, 1, (self.rows, S)).astype(np.float32)
        self.hist = (rng.random((Q, T)) ** 2 * S).astype(np.int32)
        self.lens = rng.integers(0, T + 1, Q).astype(np.int32)
        self.rep = rng.uniform(0.5, 2, Q).astype(np.float32)
        self.pre = rng.uniform(-1, 1, Q).astype(np.float32)
        self.frq = rng.uniform(0, 1, Q).astype(np.float32)

    def x(self):
        return self.t.float().numpy()

    def run(self, device_scores=None, stream=None, want_scores=True):
        import torch
        from paper_2302_06126_amd.policy import Constrain
        Q, S = self.t.shape
        d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        call = Constrain(Q, S, dtype=self.t.dtype, want_scores=want_scores)
        out = call(self.t.cuda() if device_scores is None else device_scores, allow=d(self.allow.view(np.int32)),
                   bias=d(self.bias), history=d(self.hist), history_len=d(self.lens), repetition=d(self.rep),
                   presence=d(self.pre), frequency=d(self.frq), stream=stream)
        return [o.float().cpu().numpy() if o.dtype == torch.bfloat16 else o.cpu().numpy() for o in out]

    def want(self):
        y, _ = R.constrained(self.x(), self.allow, self.bias, self.hist, self.lens, self.rep, self.pre, self.frq)
        return y


def _compare(torch, case, out):
    y = case.want()
    p, at, best = R.priors(y)
    _check_prior(out[0], p, y)
    assert np.array_equal(out[1], at)
    assert np.array_equal(out[2], best.astype(np.float32), equal_nan=True)
    if len(out) > 3:
        ref = _bf16(torch, y).float().numpy() if case.t.dtype == torch.bfloat16 else y
        assert np.array_equal(out[3], ref, equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", SIZES)
def test_constrain_sizes(torch, S, dtype):
    _say(f"[constrain] S={S} {dtype}")
    for Q, per_row in ((1, True), (7, True), (13, False)):
        case = _Case(S * 10 + Q, Q, S, dtype, per_row, T=1 if S % 2 else 40)
        _compare(torch, case, case.run())


@pytest.mark.parametrize("S", [60, 300, 9001, 20001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_constrain_what_stands_in_masked_places(torch, S, dtype):
    _say(f"[constrain] masked places S={S} {dtype}")
    case = _Case(S, 12, S, dtype)
    t, allow = case.t, case.allow.copy()
    allow[0] = 0                                     # nothing left
    allow[1] = 0
    allow[1, S // 32] = np.uint32(1) << np.uint32(S % 32 - 1 if S % 32 else 0)   # one left
    bits = ((allow[:, np.arange(S) // 32] >> (np.arange(S) % 32).astype(np.uint32)) & 1).astype(bool)
    x = t.float().numpy().copy()
    rng = np.random.default_rng(S)
    junk = rng.choice(np.array([np.nan, np.inf, -np.inf, 3e38, -3e38], np.float32), x.shape)
    x = np.where(bits, x, junk)
    x[2, bits[2]] = -np.inf                          # all that is allowed is -inf already
    case.t, case.allow = torch.from_numpy(x).to(t.dtype), allow
    case.bias[3] = np.finfo(np.float32).min          # the lowest value in place of -inf
    case.bias[4, bits[4]] = -np.inf                  # forbidden by the bias
    case.rep[5] = 1e-30                              # (overflows to infinities)
    out = case.run()
    _compare(torch, case, out)
    for q in (0, 2, 4):
        assert out[1][q] == -1 and np.isneginf(out[2][q]) and not out[0][q].any()
    assert np.isfinite(out[0][1]).all() and out[0][1].max() == 1.0


@pytest.mark.parametrize("S", [50, 700, 5000, 10000, 20000])
def test_constrain_nan_and_infinity_where_allowed(torch, S):
    from paper_2302_06126_amd.policy import Constrain
    x = np.random.default_rng(S).normal(0, 1, (5, S)).astype(np.float32)
    x[1, S // 2] = np.nan
    x[2, S - 1] = np.nan
    x[3, S // 3] = np.inf
    x[4] = np.nan
    prior, at, best = Constrain(5, S)(torch.from_numpy(x).cuda())
    prior, at, best = prior.cpu().numpy(), at.cpu().numpy(), best.cpu().numpy()
    p, _, _ = R.priors(x[:1])
    _check_prior(prior[:1], p, x[:1])
    assert at.tolist() == [int(x[0].argmax()), -1, -1, S // 3, -1]
    assert np.isnan(prior[1:]).all()
    assert best[0] == x[0].max() and np.isnan(best[[1, 2, 4]]).all() and best[3] == np.inf


def test_constrain_ties_go_to_the_lowest_slice(torch):
    from paper_2302_06126_amd.policy import Constrain
    for S in (64, 200, 1000, 3000, 6000, 30000):
        x = torch.zeros(3, S, device="cuda", dtype=torch.bfloat16)
        x[1, S // 2:] = 1.0
        x[2, -1] = x[2, S // 3] = 2.0
        _, at, _ = Constrain(3, S, dtype=torch.bfloat16)(x)
        assert at.tolist() == [0, S // 2, S // 3], S


@pytest.mark.parametrize("S", [60, 500, 4500, 9000, 20000])
def test_constrain_history_edges(torch, S):
    """Ids out of range, lengths of zero, below zero and above the rows, the same
    id throughout, a history longer than the row."""
    case = _Case(S + 1, 6, S, "f32", T=12000)
    rng = np.random.default_rng(S)
    case.hist = rng.integers(-3, S + 3, (6, 12000)).astype(np.int32)
    case.hist[1] = S - 1
    case.hist[2, :2] = [np.iinfo(np.int32).min, np.iinfo(np.int32).max]
    case.lens = np.array([12000, 12000, 2, 0, -5, 1 << 30], np.int32)
    _compare(torch, case, case.run())
    # one history for every query, all of it
    from paper_2302_06126_amd.policy import Constrain
    h = case.hist[5:6, :77]
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    out = Constrain(6, S)(case.t.cuda(), history=d(h), presence=d(case.pre))
    y, _ = R.constrained(case.x(), history=h, pre=case.pre)
    p, at, best = R.priors(y)
    _check_prior(out[0].cpu().numpy(), p, y)
    assert np.array_equal(out[1].cpu().numpy(), at)
    # a history of no columns
    a = Constrain(6, S)(case.t.cuda(), history=d(np.zeros((6, 0), np.int32)))
    b = Constrain(6, S)(case.t.cuda())
    assert all(torch.equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", [37, 256, 1500, 8195, 20001])
def test_constrain_rows_anywhere(torch, S, dtype):
    """Rows of a wider tensor that start at odd elements: the same bits."""
    case = _Case(S + 7, 9, S, dtype)
    base = case.run()
    wide = torch.full((9, S + 13), 7.0, dtype=case.t.dtype, device="cuda")
    wide[:, 5:5 + S] = case.t.cuda()
    out = case.run(device_scores=wide[:, 5:5 + S])
    assert np.array_equal(out[1], base[1]) and np.array_equal(out[3], base[3])
    assert np.array_equal(out[0], base[0]) and np.array_equal(out[2], base[2])


def test_constrain_in_place_and_rows_behind_the_last(torch):
    import paper_2302_06126_amd as P
    from paper_2302_06126_amd._abi import check, tag_constraints
    lib = P._abi.load()
    for S, dtype in ((60, torch.float32), (256, torch.bfloat16), (3000, torch.float32), (8500, torch.bfloat16),
                     (9000, torch.float32), (20000, torch.float32), (20001, torch.bfloat16)):
        case = _Case(S, 5, S, "bf16" if dtype == torch.bfloat16 else "f32")
        x = torch.full((8, S + 4), 9.0, dtype=dtype, device="cuda")
        x[:5, :S] = case.t.cuda()
        prior = torch.full((8, S + 8), 9.0, device="cuda")
        at = torch.full((8,), 9, dtype=torch.int32, device="cuda")
        best = torch.full((8,), 9.0, device="cuda")
        bias = torch.from_numpy(case.bias).cuda()
        b = C.c_size_t(0)
        check(lib.tag_constrain_workspace(5, S, C.byref(b)), "ws")
        ws = torch.full((b.value + 16,), 255, dtype=torch.uint8, device="cuda")
        c = tag_constraints()
        c.bias, c.bias_stride = bias.data_ptr(), S
        check(lib.tag_constrain(5, S, 1 if dtype == torch.bfloat16 else 0, x.data_ptr(), S + 4, C.byref(c),
                                x.data_ptr(), S + 4, prior.data_ptr(), S + 8, at.data_ptr(), best.data_ptr(),
                                ws.data_ptr(), b.value, torch.cuda.current_stream().cuda_stream), "tag_constrain")
        y, _ = R.constrained(case.x(), bias=case.bias)
        p, want, _ = R.priors(y)
        ref = torch.from_numpy(y).to(dtype)
        assert torch.equal(x[:5, :S].cpu(), ref)
        _check_prior(prior[:5, :S].cpu().numpy(), p, y)
        assert at[:5].tolist() == want.tolist()
        assert (x[5:] == 9).all() and (x[:, S:] == 9).all() and (prior[5:] == 9).all() and (prior[:, S:] == 9).all()
        assert (at[5:] == 9).all() and (best[5:] == 9).all() and (ws[b.value:] == 255).all()


def test_constrain_python_refusals(torch):
    from paper_2302_06126_amd.policy import Balance, Constrain
    call = Constrain(4, 50)
    x = torch.zeros(4, 50, device="cuda")
    bad = [dict(scores=x.to(torch.bfloat16)), dict(scores=x.cpu()), dict(scores=x[:3]), dict(scores=x[0]),
           dict(scores=torch.zeros(50, 4, device="cuda").t()), dict(allow=torch.zeros(4, 3, dtype=torch.int32, device="cuda")),
           dict(allow=torch.zeros(4, 2, device="cuda")), dict(bias=x.double()), dict(bias=x[:2]),
           dict(history=torch.zeros(4, 3, device="cuda")), dict(history=torch.zeros(3, 3, dtype=torch.int32, device="cuda")),
           dict(presence=torch.zeros(4, device="cuda")), dict(history_len=torch.zeros(4, dtype=torch.int32, device="cuda")),
           dict(history=torch.zeros(4, 3, dtype=torch.int32, device="cuda"), repetition=torch.zeros(3, device="cuda"))]
    for kw in bad:
        kw.setdefault("scores", x)
        with pytest.raises(ValueError):
            call(**kw)
    for f in (lambda: Constrain(4, 50, dtype=torch.float16), lambda: Constrain(4, 50, device="cpu")):
        with pytest.raises(ValueError):
            f()
    bal = Balance(np.ones(50, np.uint64), 2, 4)
    for kw in (dict(scores=x[:2]), dict(scores=x, use=torch.ones(4, device="cuda")),
               dict(scores=x, use=torch.ones(3, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            bal(**kw)


# -------------------------------------------------------------------- balance
def _bal_case(seed, Q, S, M, dtype, torch):
    rng = np.random.default_rng((2302, 6, seed))
    x = (rng.normal(0, 1.5, (Q, S)) + rng.normal(0, 1.5, S)).astype(np.float32)
    t = torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    masks = rng.integers(0, 1 << 63, S, dtype=np.uint64) & rng.integers(0, 1 << 63, S, dtype=np.uint64)
    masks |= rng.integers(0, 2, S).astype(np.uint64) << np.uint64(63)
    use = rng.random(Q) < 0.9
    return t, masks, use


def _check_balance(t, masks, M, coef, use, bal, bf16):
    x = t.float().cpu().numpy()
    loss, grad, count, load, h = R.balance(x, masks, M, coef, use)
    assert np.array_equal(bal.count.cpu().numpy(), count)
    assert np.all(np.abs(bal.load.cpu().numpy() - load) <= 1.01 * R.EPS * load)
    H = np.abs(h - load.sum() / M).max(initial=0.0)
    n = max(1, int((np.asarray(use) if use is not None else np.ones(len(x))).sum()))
    steps = 4 * 88 + 160
    got = float(bal.loss.item())
    assert abs(got - loss) <= coef * M * H * steps * R.EPS + 2 * R.EPS * abs(loss), (got, loss)
    with np.errstate(invalid="ignore", over="ignore"):
        e = np.exp(x.astype(np.float64) - x.max(axis=1, keepdims=True))
    p = e / e.sum(axis=1, keepdims=True)
    tol = coef * M / n * p * 2 * H * steps * R.EPS + 2.0 ** -125
    g = bal.grad.float().cpu().numpy().astype(np.float64)
    if bf16:
        tol = tol + np.abs(grad) * 2.0 ** -8
    assert np.all(np.abs(g - grad) <= tol), float((np.abs(g - grad) / tol).max())
    if use is not None:
        assert not g[~np.asarray(use, bool)].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", [1, 2, 31, 60, 64, 65, 255, 256, 257, 1024, 1025, 4096, 4097, 16383, 16384])
def test_balance_sizes(torch, S, dtype):
    from paper_2302_06126_amd.policy import Balance
    for Q, M in ((1, 1), (5, 64), (37, 7)):
        _say(f"[balance] S={S} Q={Q} M={M} {dtype}")
        t, masks, use = _bal_case(S * 100 + Q, Q, S, M, dtype, torch)
        use = None if Q == 1 else use
        bal = Balance(masks, M, Q, dtype=t.dtype)
        bal(t.cuda(), 0.02, use=None if use is None else torch.from_numpy(use).cuda())
        _check_balance(t, masks, M, 0.02, use, bal, dtype == "bf16")


@pytest.mark.parametrize("Q,S,M", [(9000, 60, 4), (20011, 256, 64), (5000, 700, 16), (3001, 4096, 32)])
def test_balance_many_rows(torch, Q, S, M):
    """More rows than blocks walk at once; repeated calls give the same bits."""
    from paper_2302_06126_amd.policy import Balance
    _say(f"[balance] Q={Q} S={S} M={M}")
    t, masks, use = _bal_case(Q + S, Q, S, M, "f32", torch)
    bal = Balance(masks, M, Q)
    u, x = torch.from_numpy(use.astype(np.uint8)).cuda(), t.cuda()
    bal(x, 0.01, use=u)
    _check_balance(t, masks, M, 0.01, use, bal, False)
    first = [v.clone() for v in (bal.loss, bal.grad, bal.count, bal.load)]
    bal.ws.fill_(255)
    bal(x, 0.01, use=u)
    assert all(torch.equal(a, b) for a, b in zip(first, (bal.loss, bal.grad, bal.count, bal.load)))


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("S,M", [(60, 8), (250, 64), (1111, 49), (9000, 30)])
def test_balance_of_one_row(torch, S, M, seed):
    """One query's gradient is small differences of h, most of which are far
    below that of the slice it chose.  With h' = h less the mean load, in units
    of 2^-24: h' and p'h rounded (1 each of |h'| and of their row's mean |h'|, the
    sum's terms 3 for e^x and 1 for the product, its additions 2 by their root),
    their difference, and 8 for p, the scale and the result."""
    from paper_2302_06126_amd.policy import Balance
    rng = np.random.default_rng((2302, seed, S, M))
    x = rng.normal(0, 2, (1, S)).astype(np.float32)
    masks = np.zeros(S, np.uint64)
    for _ in range(3):   # up to three devices of a slice
        masks |= np.uint64(1) << rng.integers(0, M, S, dtype=np.uint64)
    bal = Balance(masks, M, 1)
    loss = bal(torch.from_numpy(x).cuda(), 0.01).item()
    want, grad, count, load, h = R.balance(x, masks, M, 0.01)
    p = np.exp(x[0].astype(np.float64) - x.max())
    p /= p.sum()
    off = np.abs(h - load.sum() / M)
    tol = R.EPS * (0.01 * M * p * (off + 8 * (p @ off)) + 8 * np.abs(grad[0]))
    err = np.abs(bal.grad.cpu().numpy()[0] - grad[0])
    _say(f"   {np.linalg.norm(err) / np.linalg.norm(grad):.2e} of the gradient, {(err / tol).max():.2f} of the tolerance")
    assert np.all(err <= tol + 2.0 ** -125) and abs(loss - want) <= 8 * R.EPS * want


@pytest.mark.parametrize("S", [50, 300, 2000, 5000])
def test_balance_edges(torch, S):
    from paper_2302_06126_amd.policy import Balance
    t, masks, _ = _bal_case(S, 8, S, 6, "f32", torch)
    masks[: S // 2] = 0                              # slices without a device
    masks[S // 2:] |= np.uint64(1 << 40)             # bits past the devices
    x = t.cuda()
    bal = Balance(masks, 6, 8)
    # rows left out may hold anything; rows of -inf are left out
    x[2] = float("nan")
    x[5] = float("-inf")
    x[6, ::2] = float("-inf")
    use = torch.tensor([1, 1, 0, 1, 1, 1, 1, 1], dtype=torch.uint8, device="cuda")
    bal(x, 0.5, use=use)
    ref = x.cpu().numpy().astype(np.float64)
    ref[2] = -np.inf
    loss, grad, count, load, h = R.balance(ref, masks, 6, 0.5)
    assert count.sum() == 6 and np.array_equal(bal.count.cpu().numpy(), count)
    assert abs(bal.loss.item() - loss) <= 1e-5 * abs(loss) and not bal.grad[2].any() and not bal.grad[5].any()
    assert np.abs(bal.grad.cpu().numpy() - grad).max() <= 1e-5 * np.abs(grad).max()
    # none used
    bal(x, 0.5, use=torch.zeros(8, dtype=torch.bool, device="cuda"))
    assert bal.loss.item() == 0 and not bal.grad.any() and not bal.count.any() and not bal.load.any()
    # a NaN or an infinity in a used row
    for v in (float("nan"), float("inf")):
        y = t.cuda()
        y[3, S // 2] = v
        bal(y, 0.5)
        assert np.isnan(bal.loss.item()) and torch.isnan(bal.grad[3]).all()
        assert torch.isfinite(bal.grad[[0, 1, 2, 4, 5, 6, 7]]).all()
        assert int(bal.count.sum()) == (7 if v != v else 8)


@pytest.mark.parametrize("S", [61, 1000, 4500])
def test_balance_rows_anywhere_and_added_gradients(torch, S):
    import paper_2302_06126_amd as P
    from paper_2302_06126_amd._abi import check
    from paper_2302_06126_amd.policy import Balance
    t, masks, use = _bal_case(S, 11, S, 9, "f32", torch)
    bal = Balance(masks, 9, 11)
    u = torch.from_numpy(use).cuda()
    bal(t.cuda(), 0.1, use=u)
    wide = torch.full((14, S + 7), 3.0, device="cuda")
    wide[:11, 3:3 + S] = t.cuda()
    other = Balance(masks, 9, 11)
    other(wide[:11, 3:3 + S], 0.1, use=u)
    for a, b in zip((bal.loss, bal.grad, bal.count, bal.load), (other.loss, other.grad, other.count, other.load)):
        assert torch.equal(a, b)
    g = torch.randn(14, S + 2, device="cuda")
    was = g.clone()
    check(P._abi.load().tag_balance(11, S, 0, wide[:, 3:].data_ptr(), S + 7, bal.masks.data_ptr(), 9, u.data_ptr(), 0.1,
                                    g.data_ptr(), S + 2, 1, other.loss.data_ptr(), other.count.data_ptr(),
                                    other.load.data_ptr(), other.ws.data_ptr(), other.ws_bytes,
                                    torch.cuda.current_stream().cuda_stream), "tag_balance")
    assert torch.equal(g[:11, :S], was[:11, :S] + bal.grad) and torch.equal(g[11:], was[11:])
    assert torch.equal(g[:, S:], was[:, S:]) and torch.equal(other.loss, bal.loss)


# ------------------------------------------------------- streams, graphs, chain
def test_side_streams_and_captured_graphs(torch):
    """Two objects captured into two graphs, replayed in turn on new inputs with
    eager calls between, on a stream of their own."""
    from paper_2302_06126_amd.policy import Balance, Constrain
    s = torch.cuda.Stream()
    objs = []
    for S, Q in ((256, 300), (9000, 5), (20000, 7)):
        t, masks, _ = _bal_case(S, Q, S, 8, "f32", torch)
        S_b = min(S, 256)
        x = t.cuda()
        con, bal = Constrain(Q, S), Balance(masks[:S_b], 8, Q)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            con(x)
            bal(x[:, :S_b])
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            con(x)
            bal(x[:, :S_b])
        objs.append((x, con, bal, g, masks[:S_b], S_b))
    for i in range(3):
        for x, con, bal, g, masks, S_b in objs:
            new = torch.randn(x.shape, device="cuda")
            x.copy_(new)
            g.replay()
            torch.cuda.synchronize()
            got = [v.clone() for v in (con.prior, con.argmax, con.best, bal.loss, bal.grad, bal.count, bal.load)]
            eager_c, eager_b = Constrain(*x.shape), Balance(masks, 8, x.shape[0])
            eager_c(new)
            eager_b(new[:, :S_b])
            want = (eager_c.prior, eager_c.argmax, eager_c.best, eager_b.loss, eager_b.grad, eager_b.count, eager_b.load)
            assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    # an explicit stream
    x, con, bal, _, masks, S_b = objs[0]
    s.wait_stream(torch.cuda.current_stream())
    con(x, stream=s)
    bal(x, stream=s)
    s.synchronize()
    assert torch.equal(con.prior, objs[0][1].prior)


@pytest.mark.parametrize("f,H,S,per", [(64, 64, 60, 3), (128, 32, 101, 5), (64, 0, 33, 2), (64, 16, 200, 600)])
def test_scores_then_constraints_then_balance(torch, f, H, S, per):
    """The decision head's raw scores through both operators: without
    constraints the head's own priors; the decisions under masks lie in them;
    the balance loss of what is left."""
    import paper_2302_06126_amd as P
    import synth
    from paper_2302_06126_amd.policy import Balance, Constrain
    R_, n_op, n_dev = 16, 40, 6
    rng = np.random.default_rng((2302, 8, f, S))
    topo = synth.random_topology(31, n_op, n_dev, 2 * n_op)
    g = P.Graph([topo])
    m = P.Model(synth.make_weights(f, 4, 1, 42, H, bias_scale=0.5, seed_extra=1), f=f, heads=4, layers=1, f_op=42,
                dec_hidden=H)
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    E_op = d(rng.uniform(0, 1, (R_, n_op, f)).astype(np.float32))
    E_dev = d(rng.uniform(0, 1, (R_, n_dev, f)).astype(np.float32))
    masks, opts = synth.make_slices("cnn", n_dev, S)
    q_rep = np.repeat(np.arange(R_), per).astype(np.int32)
    q_op = rng.integers(0, n_op, len(q_rep)).astype(np.int32)
    q_rep[-1] = R_   # an out-of-range query
    Q = len(q_rep)
    _say(f"[chain] f={f} H={H} S={S} Q={Q}")
    dec = P.Decide(g, m, R_, masks, opts, q_rep, np.zeros_like(q_op), q_op)
    dec(E_op, E_dev)
    res = dec.results()
    x = dec.scores(E_op, E_dev)
    assert torch.equal(x, P.scores(g, m, E_op, E_dev, masks, opts, q_rep, np.zeros_like(q_op), q_op))
    assert torch.isneginf(x[-1]).all() and torch.isfinite(x[:-1]).all()
    assert np.array_equal(dec.results()["prior"], res["prior"])   # (the head's outputs are left alone)
    con = Constrain(Q, S, want_scores=True)
    prior, at, best, y = con(x)
    assert np.array_equal(at.cpu().numpy(), res["argmax"]) and np.array_equal(best[:-1].cpu().numpy(), res["best"][:-1])
    # both are softmaxes of the same scores: the head's exponentials are rounded in x log2(e), 88 half steps at most
    assert np.all(np.abs(prior.cpu().numpy() - res["prior"]) <= (4 * 88 + 128) * R.EPS * res["prior"] + 2.0 ** -125)
    allow = _words(rng, Q, S, 0.4)
    allow[3] = 0
    prior, at, best, y = con(x, allow=d(allow.view(np.int32)))
    want, _ = R.constrained(x.cpu().numpy(), allow)
    assert np.array_equal(y.cpu().numpy(), want) and np.array_equal(at.cpu().numpy(), R.priors(want)[1])
    bal = Balance(masks, n_dev, Q)
    bal(y, 0.1)
    loss, grad, count, load, h = R.balance(want, masks, n_dev, 0.1)
    assert np.array_equal(bal.count.cpu().numpy(), count) and count.sum() == int((at >= 0).sum())
    assert abs(bal.loss.item() - loss) <= 1e-5 * loss
    assert np.abs(bal.grad.cpu().numpy() - grad).max() <= 1e-5 * np.abs(grad).max()
    g.close()
