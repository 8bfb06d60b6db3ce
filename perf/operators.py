"""The policy and optimiser operators as cases that can be timed.

Next to the decision head and the training step stand four operators, which a
case names by "op":

  constrain      scores [Q, S] of the decision head under what a caller knows
                 and the network does not: slices that are not allowed (a bit
                 mask), a bias per slice, penalties for slices that the query's
                 history took already; then the softmax and the argmax
  balance        the loss that spreads the decisions over the devices, the
                 count of each slice, each device's load, and the gradient with
                 respect to the scores
  orthogonalise  Newton-Schulz products that bring a matrix's singular values
                 near one (five steps of the quintic)
  muon           the optimiser step around it: momentum, orthogonalised update
                 of every weight matrix, momentum SGD for the rest

Where ``own`` is false, ``run`` computes them from elementary torch operations;
where it is true, by the framework's calls.  ``exact`` restates them in 64 bits.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

STEPS, COEF, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
MOMENTUM, LR, DECAY = 0.95, 0.02, 0.01
F_OP, F_DEV = 42, 8


def _constrain(name, q, s, history, dtype, rows, scores):
    """history: longest history; rows: masks and biases of each query (else shared); scores: the constrained scores
    are wanted too."""
    return dict(name=name, op="constrain", q=q, s=s, history=history, dtype=dtype, rows=rows, scores=scores)


def _balance(name, q, s, devices, dtype):
    return dict(name=name, op="balance", q=q, s=s, devices=devices, dtype=dtype)


def _ortho(name, count, rows, cols, dtype):
    return dict(name=name, op="orthogonalise", count=count, rows=rows, cols=cols, dtype=dtype)


def _muon(name, f, layers, hidden):
    return dict(name=name, op="muon", f=f, layers=layers, hidden=hidden)


def listed():
    return [
        # one query of the 200-op graph: what a single look-up of the priors pays
        _constrain("constrain_one", 1, 60, 20, "f32", False, False),
        # a group of every candidate of the convolutional network's graph, with masks of its own for each query
        _constrain("constrain_cnn", 1932, 256, 60, "f32", True, True),
        # a whole group of every candidate of the large topology, scores kept in 16 bits
        _constrain("constrain_large_bf16", 42496, 256, 60, "bf16", True, True),
        # every placement of 16 devices with each option
        _constrain("constrain_full", 64, 262140, 60, "f32", True, False),
        # a small round on four devices
        _balance("balance_small", 64, 60, 4, "f32"),
        # a training batch of wide slice tables in 16 bits
        _balance("balance_wide_bf16", 2048, 4096, 32, "bf16"),
        # the large topology: 42,496 queries of 64 devices
        _balance("balance_large", 42496, 256, 64, "f32"),
        # one small weight matrix (the op encoder at width 64)
        _ortho("orthogonalise_small", 1, 64, 42, "f32"),
        # a wide weight matrix in 32 bits
        _ortho("orthogonalise_2048", 1, 2048, 2048, "f32"),
        # four tall matrices in 16 bits
        _ortho("orthogonalise_tall_bf16", 4, 4096, 1024, "bf16"),
        # every parameter of the convolutional network's model
        _muon("muon_cnn", 128, 3, 128),
        # every parameter of the large topology's model
        _muon("muon_large", 256, 4, 256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["constrain", "constrain", "constrain", "balance", "balance", "orthogonalise", "orthogonalise",
                     "muon"])
    dtype = rng.choice(["f32", "f32", "bf16"])
    if op == "constrain":
        s = _log_int(rng, 2, 262140)
        c = _constrain("", _log_int(rng, 1, max(1, min(42496, 8_000_000 // s))), s, _log_int(rng, 1, 512), dtype,
                       rng.random() < 0.6, rng.random() < 0.5)
    elif op == "balance":
        s = _log_int(rng, 2, 16384)
        c = _balance("", _log_int(rng, 1, max(1, min(42496, 8_000_000 // s))), s,
                     rng.choice([rng.randint(2, 16), rng.randint(17, 64)]), dtype)
    elif op == "orthogonalise":
        rows, cols = _log_int(rng, 8, 2048), _log_int(rng, 8, 2048)
        c = _ortho("", _log_int(rng, 1, max(1, min(64, 4_000_000 // (rows * cols)))), rows, cols, dtype)
    else:
        c = _muon("", rng.choice([64, 128, 256]), rng.randint(1, 6), _log_int(rng, 16, 512))
    del c["name"]
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _masks(case, rng):
    """Slice table: placements on one to eight devices."""
    m, s = case["devices"], case["s"]
    r = rng.integers(1, min(8, m) + 1, size=s)
    rank = np.argsort(np.argsort(rng.random((s, m)), axis=1), axis=1)
    return ((rank < r[:, None]).astype(np.uint64) << np.arange(m, dtype=np.uint64)[None, :]).sum(axis=1).astype(np.uint64)


def _gradient(gen, dev, *shape):
    """What gradients look like: a few strong directions over a floor of noise."""
    count, rows, cols = shape
    r = max(1, min(rows, cols) // 8)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=dev)
    strong = torch.matmul(rnd(count, rows, r) / torch.arange(1, r + 1, device=dev).sqrt(), rnd(count, r, cols))
    return 1e-3 * (strong / math.sqrt(r) + 0.3 * rnd(count, rows, cols))


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rng = np.random.default_rng((seed, 29))
    rnd = lambda *s: torch.rand(*s, generator=gen, device=dev)
    s = SimpleNamespace(case=case, op=case["op"])
    if s.op == "constrain":
        q, n, t = case["q"], case["s"], case["history"]
        words, rows = (n + 31) // 32, q if case["rows"] else 1
        s.scores = (2.0 * torch.randn(q, n, generator=gen, device=dev)).to(_type(case))
        # about three slices in four fit the devices' memory; one row in sixteen has none left
        bits = torch.randint(0, 1 << 32, (3, rows, words), generator=gen, device=dev, dtype=torch.int64)
        allow = (bits[0] | bits[1]) * (torch.rand(rows, 1, generator=gen, device=dev) >= (1 / 16 if rows > 1 else 0))
        s.allow = torch.where(allow >= 1 << 31, allow - (1 << 32), allow).to(torch.int32)
        s.bias = 0.5 * torch.randn(rows, n, generator=gen, device=dev)
        s.history = (rnd(q, t) ** 3 * n).to(torch.int32).clamp_(max=n - 1)   # (some slices again and again)
        s.length = (rnd(q) * (t + 1)).to(torch.int32).clamp_(max=t)
        s.repetition, s.presence, s.frequency = 1.0 + rnd(q), rnd(q), 0.5 * rnd(q)
        if own:
            from paper_2302_06126_amd.policy import Constrain
            s.call = Constrain(q, n, dtype=_type(case), device=dev, want_scores=case["scores"])
    elif s.op == "balance":
        q, n = case["q"], case["s"]
        lean = torch.randn(1, n, generator=gen, device=dev)   # (what the network prefers everywhere)
        s.scores = (1.5 * (torch.randn(q, n, generator=gen, device=dev) + lean)).to(_type(case))
        s.use = (rnd(q) >= 0.05).to(torch.uint8)              # padded queries
        s.masks = _masks(case, rng)
        s.table = torch.from_numpy(s.masks.view(np.int64)).to(dev)
        s.coef = 0.01
        if own:
            from paper_2302_06126_amd.policy import Balance
            s.call = Balance(s.masks, case["devices"], q, dtype=_type(case), device=dev)
    elif s.op == "orthogonalise":
        s.x = _gradient(gen, dev, case["count"], case["rows"], case["cols"]).to(_type(case))
        if own:
            from paper_2302_06126_amd.optim import Orthogonalise
            s.call = Orthogonalise([(case["count"], case["rows"], case["cols"])], dtype=_type(case), device=dev,
                                   steps=STEPS, coef=COEF, eps=EPS)
    else:
        f, layers, h = case["f"], case["layers"], case["hidden"]
        shapes = [(3 * layers, f, 2 * f), (1, f, F_OP), (1, f, F_DEV), (1, h, 2 * f + 4)]
        s.w = [torch.randn(*d, generator=gen, device=dev) / math.sqrt(d[2]) for d in shapes]
        s.g = [_gradient(gen, dev, *d) for d in shapes]
        rest = 9 * layers * f + 9 * f + 2 * h + 1   # biases, attention vectors, edge encoders, readout
        s.w.append(0.1 * torch.randn(rest, generator=gen, device=dev))
        s.g.append(1e-3 * torch.randn(rest, generator=gen, device=dev))
        s.m = [MOMENTUM * _gradient(gen, dev, *d) for d in shapes]
        s.m.append(1e-3 * torch.randn(rest, generator=gen, device=dev))
        if own:
            from paper_2302_06126_amd.optim import Muon
            s.call = Muon(list(zip(s.w, s.g)), lr=LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY,
                          steps=STEPS, coef=COEF, eps=EPS, state=s.m)
    return s


# --------------------------------------------------------------------------
# the plain form
# --------------------------------------------------------------------------

def _plain_constrain(s):
    q, n = s.scores.shape
    x = s.scores.float()
    t = s.history.shape[1]
    live = (torch.arange(t, device=x.device)[None, :] < s.length[:, None]).float()
    count = torch.zeros(q, n, device=x.device).scatter_add_(1, s.history.long(), live)
    seen = count > 0
    rep = s.repetition[:, None]
    y = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    y = y - s.frequency[:, None] * count - s.presence[:, None] * seen + s.bias
    at = torch.arange(n, device=x.device)
    allowed = (s.allow[:, at // 32] >> (at % 32)) & 1
    y = torch.where(allowed.bool(), y, torch.full_like(y, -math.inf))
    best, argmax = y.max(dim=1)
    argmax = torch.where(y == best[:, None], at[None, :], n).min(dim=1).values   # ties: the lowest index
    some = best > -math.inf
    e = torch.exp(y - torch.where(some, best, torch.zeros_like(best))[:, None])
    prior = e / e.sum(dim=1, keepdim=True).clamp_min(1e-30)
    argmax = torch.where(some, argmax, torch.full_like(argmax, -1)).to(torch.int32)
    return (prior, argmax, best) + ((y.to(s.scores.dtype),) if s.case["scores"] else ())


def _shares(table, m):
    """[S, M] in 64 bits: what part of a slice's work each device does."""
    bits = ((table[:, None] >> torch.arange(m, device=table.device)) & 1).double()
    return bits / bits.sum(dim=1, keepdim=True).clamp_min(1)


def _plain_balance(s):
    q, n = s.scores.shape
    m = s.case["devices"]
    x = s.scores.float()
    use = s.use.bool()
    best = x.max(dim=1, keepdim=True).values
    at = torch.arange(n, device=x.device)
    argmax = torch.where(x == best, at[None, :], n).min(dim=1).values
    count = torch.zeros(n, dtype=torch.int32, device=x.device).scatter_add_(0, argmax, s.use.to(torch.int32))
    rows = use.sum().clamp_min(1)
    shares = _shares(s.table, m)
    load = (count.double()[:, None] * shares).sum(dim=0) / rows
    h = (shares * load).sum(dim=1)
    e = torch.exp(x - best)
    p = e / e.sum(dim=1, keepdim=True)
    off = (h - h.mean()).float()   # (the mean taken off in 64 bits: it cancels)
    mean = (p * off).sum(dim=1, keepdim=True)
    scale = s.coef * m / rows.float()
    grad = torch.where(use[:, None], scale * p * (off - mean), torch.zeros_like(p))
    loss = scale.double() * torch.where(use, mean[:, 0].double(), 0.0).sum() + s.coef * m * h.mean() * (rows > 0)
    return loss.float().reshape(1), grad.to(s.scores.dtype), count, load.float()


def _plain_newton_schulz(g):
    x = g.transpose(1, 2) if g.shape[1] > g.shape[2] else g
    x = x / (x.double().square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS).float()
    a, b, c = COEF
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return x.transpose(1, 2) if g.shape[1] > g.shape[2] else x


def _plain_muon(w, g, m):
    m.mul_(MOMENTUM).add_(g)
    u = g + MOMENTUM * m
    w.mul_(1.0 - LR * DECAY)
    if w.dim() == 3:
        u = _plain_newton_schulz(u) * math.sqrt(max(1.0, w.shape[1] / w.shape[2]))
    w.sub_(u, alpha=LR)


def run(s):
    if own:
        if s.op == "constrain":
            return s.call(s.scores, allow=s.allow, bias=s.bias, history=s.history, history_len=s.length,
                          repetition=s.repetition, presence=s.presence, frequency=s.frequency)
        if s.op == "balance":
            loss = s.call(s.scores, s.coef, use=s.use)
            return loss, s.call.grad, s.call.count, s.call.load
        if s.op == "orthogonalise":
            return s.call([s.x])
        s.call.step()
        return s.w, s.m
    if s.op == "constrain":
        return _plain_constrain(s)
    if s.op == "balance":
        return _plain_balance(s)
    if s.op == "orthogonalise":
        return [_plain_newton_schulz(s.x.float()).to(s.x.dtype).contiguous()]
    for w, g, m in zip(s.w, s.g, s.m):
        _plain_muon(w, g, m)
    return s.w, s.m


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def _ortho_flops(count, rows, cols):
    """The symmetric products take their half."""
    n, m = min(rows, cols), max(rows, cols)
    return float(count) * STEPS * (n * n * m + n * n * n + 2.0 * n * n * m)


def work(case):
    b = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "constrain":
        q, n = case["q"], case["s"]
        rows = q if case["rows"] else 1
        return {"bytes": q * n * (b + 4.0 + (b if case["scores"] else 0)) + rows * n * 4.125 + q * case["history"] * 4.0
                + q * 24.0, "flops": 8.0 * q * n}
    if case["op"] == "balance":
        q, n = case["q"], case["s"]
        return {"bytes": q * n * 2.0 * b + n * 12.0 + q, "flops": 8.0 * q * n}
    if case["op"] == "orthogonalise":
        return {"bytes": 2.0 * b * case["count"] * case["rows"] * case["cols"],
                "flops": _ortho_flops(case["count"], case["rows"], case["cols"])}
    f, layers, h = case["f"], case["layers"], case["hidden"]
    shapes = [(3 * layers, f, 2 * f), (1, f, F_OP), (1, f, F_DEV), (1, h, 2 * f + 4)]
    values = sum(c * r * k for c, r, k in shapes) + 9 * layers * f + 9 * f + 2 * h + 1
    return {"bytes": 20.0 * values, "flops": sum(_ortho_flops(*d) for d in shapes) + 6.0 * values}


# --------------------------------------------------------------------------
# 64 bits
# --------------------------------------------------------------------------

def _exact_constrain(s):
    """By each query's own list of slices, on the host."""
    x = s.scores.double().cpu().numpy()
    q, n = x.shape
    words = s.allow.cpu().numpy().view(np.uint32)
    allowed = np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:, :n].astype(bool)
    bias = s.bias.double().cpu().numpy()
    hist, length = s.history.cpu().numpy(), s.length.cpu().numpy()
    rep, pre, frq = (v.double().cpu().numpy() for v in (s.repetition, s.presence, s.frequency))
    for i in range(q):
        a, c = np.unique(hist[i, :length[i]], return_counts=True)
        v = x[i, a]
        x[i, a] = np.where(v > 0, v / rep[i], v * rep[i]) - pre[i] - frq[i] * c
    x += bias
    x[~np.broadcast_to(allowed, x.shape)] = -np.inf
    best = x.max(axis=1)
    none = np.isneginf(best)
    argmax = np.where(none, -1, x.argmax(axis=1)).astype(np.int32)
    z = np.exp(x - np.where(none, 0.0, best)[:, None])
    prior = z / np.where(none, 1.0, z.sum(axis=1))[:, None]
    return (prior, argmax, best) + ((x,) if s.case["scores"] else ())


def _exact_balance(s):
    x = s.scores.double()
    m, use = s.case["devices"], s.use.bool()
    n = int(use.sum())
    p = torch.zeros_like(x)
    p[use] = torch.softmax(x[use], dim=1)
    count = torch.bincount(x[use].argmax(dim=1), minlength=x.shape[1])
    bits = torch.from_numpy(((s.masks[:, None] >> np.arange(m, dtype=np.uint64)) & np.uint64(1)).astype(np.float64)).to(x.device)
    share = bits / bits.sum(dim=1, keepdim=True)
    load = count.double() @ share / max(n, 1)
    worth = share @ load
    loss = s.coef * m * (load * (p.sum(dim=0) @ share)).sum() / max(n, 1)
    grad = s.coef * m / max(n, 1) * p * (worth[None, :] - (p @ worth)[:, None])
    return loss.reshape(1), grad, count.to(torch.int32), load


def _exact_newton_schulz(g):
    """In the order x (a + b k + c k k) with k = x^T x, on the narrow side."""
    x = g.double()
    wide = x.shape[1] < x.shape[2]
    x = (x.transpose(1, 2) if wide else x).contiguous()
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + EPS)
    a, b, c = COEF
    eye = torch.eye(x.shape[2], dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        k = x.transpose(1, 2).contiguous() @ x
        x = x @ (a * eye + k @ (b * eye + c * k))
    return x.transpose(1, 2).contiguous() if wide else x


def exact(case, seed):
    s = prepare(case, seed)
    if s.op == "constrain":
        return _exact_constrain(s)
    if s.op == "balance":
        return _exact_balance(s)
    if s.op == "orthogonalise":
        return [_exact_newton_schulz(s.x)]
    ws, ms = [], []
    for w, g, m in zip(s.w, s.g, s.m):
        m = MOMENTUM * m.double() + g.double()
        u = g.double() + MOMENTUM * m
        if w.dim() == 3:
            u = math.sqrt(max(1.0, w.shape[1] / w.shape[2])) * _exact_newton_schulz(u)
        ws.append((1.0 - LR * DECAY) * w.double() - LR * u)
        ms.append(m)
    return ws, ms
