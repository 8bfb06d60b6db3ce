"""Beam search and gradient clipping as cases that can be timed.

Operators of decoding and training next to the decision head, the search and the
optimiser, which a case names by "op":

  beam     one level of a beam search: n searches of V beams each, whose scores
           [n V, S] become log probabilities; the best W of the V S
           continuations with their parents and slices.  Finished beams are
           carried along, beams with a total of -inf are not there
  reorder  the beams' states (features, placement bits, paths) follow their
           parents, in place or into other tensors
  clip     the 2-norm over all gradients and, where it is above a limit, the
           gradients scaled down to it
  step     the optimiser step (momentum, orthogonalised updates) of a model's
           parameters from clipped gradients

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


def _beam(name, n, v, w, s, dtype, done):
    """n searches of v beams, w after it, s slices; done: the share of finished beams."""
    return dict(name=name, op="beam", n=n, v=v, w=w, s=s, dtype=dtype, done=done)


def _reorder(name, n, w, ops, devices, depth, links, place):
    """States of n w beams: ops x 42 and devices x 8 features, a placement bit per op and linked device, a path of depth
    groups; place: in place."""
    return dict(name=name, op="reorder", n=n, w=w, ops=ops, devices=devices, depth=depth, links=links, place=place)


def _clip(name, kind, tensors, size, dtype, limit):
    """kind "model": the parameters of a model of width `size` with `tensors` layers; "many": `tensors` tensors of 1 to
    `size` values, long rows among them; limit: of the norm, relative to it."""
    return dict(name=name, op="clip", kind=kind, tensors=tensors, size=size, dtype=dtype, limit=limit)


def _step(name, f, layers, hidden, limit):
    return dict(name=name, op="step", f=f, layers=layers, hidden=hidden, limit=limit)


def listed():
    return [
        # one level of a narrow search on the 200-op graph: what a single decision pays
        _beam("beam_one", 1, 4, 4, 60, "f32", 0.0),
        # a search as wide as the leaf batches of the convolutional network's graph
        _beam("beam_cnn", 1, 64, 64, 256, "f32", 0.0),
        # many searches at once over the large topology's slices, scores kept in 16 bits, some searches at their end
        _beam("beam_large_bf16", 2656, 16, 16, 256, "bf16", 0.1),
        # wide searches over a wide table of odd length
        _beam("beam_wide", 5, 200, 200, 4099, "f32", 0.1),
        # every placement of 16 devices with each option
        _beam("beam_full", 8, 8, 8, 262140, "f32", 0.0),
        # the states of one wide search on the convolutional network's graph, 16 devices, in place
        _reorder("reorder_cnn", 1, 64, 1200, 16, 60, 16, True),
        # the states of several searches on the large topology, from one set of buffers to the other
        _reorder("reorder_large", 8, 16, 10000, 64, 60, 16, False),
        # the gradients of the convolutional network's model
        _clip("clip_cnn", "model", 3, 128, "f32", 0.6),
        # many tensors of odd sizes, in 16 and in 32 bits
        _clip("clip_many", "many", 1200, 100000, "mixed", 0.3),
        # more than the caches hold
        _clip("clip_large", "many", 128, 16000000, "f32", 0.7),
        # a small model's optimiser step from clipped gradients
        _step("step_tiny", 64, 2, 64, 0.3),
        # every parameter of the large topology's model
        _step("step_large", 256, 4, 256, 0.6),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["beam", "beam", "beam", "reorder", "reorder", "clip", "clip", "step"])
    if op == "beam":
        w = _log_int(rng, 1, 256)
        v = rng.choice([w, w, w, 1, _log_int(rng, 1, 256)])
        s = _log_int(rng, 2, min(262140, 16_000_000 // v))
        c = _beam("", _log_int(rng, 1, max(1, min(42496 // v, 16_000_000 // (s * v)))), v, w, s,
                  rng.choice(["f32", "f32", "bf16"]), rng.choice([0.0, rng.uniform(0.0, 0.5)]))
    elif op == "reorder":
        w, ops = _log_int(rng, 1, 256), _log_int(rng, 20, 10000)
        links = rng.randint(1, 16)
        c = _reorder("", _log_int(rng, 1, max(1, 1_250_000 // (w * ops))), w, ops, rng.randint(links, 64),
                     rng.randint(1, 120), links, rng.random() < 0.6)
    elif op == "clip":
        dtype, limit = rng.choice(["f32", "bf16", "mixed"]), rng.choice([rng.uniform(0.05, 0.95), rng.uniform(0.05, 0.95), 2.0])
        if rng.random() < 0.3:
            c = _clip("", "model", rng.randint(1, 6), rng.choice([64, 128, 256]), dtype, limit)
        else:
            n = _log_int(rng, 1, 2000)
            c = _clip("", "many", n, _log_int(rng, 16, min(16_000_000, 200_000_000 // n)), dtype, limit)
    else:
        c = _step("", rng.choice([64, 128, 256]), rng.randint(1, 6), _log_int(rng, 16, 512), rng.choice([0.1, 0.5, 0.9, 2.0]))
    del c["name"]
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _model_shapes(f, layers, hidden):
    """Weight matrices and the length of everything else."""
    return [(3 * layers, f, 2 * f), (1, f, F_OP), (1, f, F_DEV), (1, hidden, 2 * f + 4)], 9 * layers * f + 9 * f + 2 * hidden + 1


def _sizes(case):
    """The tensors of a clip case: (rows, columns, row stride, bits)."""
    if case["kind"] == "model":
        mats, rest = _model_shapes(case["size"], case["tensors"], case["size"])
        shapes = [(c * r, k, k) for c, r, k in mats] + [(1, rest, rest)]
    else:
        # sizes from a stream that is the case's own, so that every seed has the same ones
        rng = np.random.default_rng((case["tensors"], case["size"], 7))
        shapes = []
        for _ in range(case["tensors"]):
            n = int(round(math.exp(rng.uniform(0.0, math.log(case["size"])))))
            rows = 1 if n < 64 or rng.random() < 0.7 else int(rng.integers(2, 33))
            cols = max(1, n // rows)
            shapes.append((rows, cols, cols if rng.random() < 0.8 else cols + int(rng.integers(1, 9))))
    bits = {"f32": [32], "bf16": [16], "mixed": [16, 16, 32]}[case["dtype"]]
    return [(r, c, t, bits[i % len(bits)]) for i, (r, c, t) in enumerate(shapes)]


def _gradient(gen, dev, *shape):
    """What gradients look like: a few strong directions over a floor of noise."""
    count, rows, cols = shape
    r = max(1, min(rows, cols) // 8)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=dev)
    strong = torch.matmul(rnd(count, rows, r) / torch.arange(1, r + 1, device=dev).sqrt(), rnd(count, r, cols))
    return 1e-3 * (strong / math.sqrt(r) + 0.3 * rnd(count, rows, cols))


def _flat(shapes, dev, double=False):
    """Tensors of the given (rows, columns, bits) as pieces of one buffer for each type, as a program that sends its
    gradients over a network keeps them; pieces start at multiples of 64 values."""
    pieces, size = [], {16: 0, 32: 0}
    for r, c, b in shapes:
        pieces.append((b, size[b]))
        size[b] += (r * c + 63) // 64 * 64
    kind = lambda b: torch.float64 if double else torch.bfloat16 if b == 16 else torch.float32
    flat = {b: torch.zeros(n, dtype=kind(b), device=dev) for b, n in size.items() if n}
    return list(flat.values()), [flat[b][at:at + r * c].view(r, c) for (r, c, _), (b, at) in zip(shapes, pieces)]


def _norm(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rnd = lambda *s: torch.rand(*s, generator=gen, device=dev)
    nrm = lambda *s: torch.randn(*s, generator=gen, device=dev)
    s = SimpleNamespace(case=case, op=case["op"])
    if s.op == "beam":
        n, v, a = case["n"], case["v"], case["s"]
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        x = 2.0 * nrm(n * v, a)
        # about one slice in four does not fit the devices' memory; a beam in 64 has none left
        x.masked_fill_(rnd(n * v, a) < 0.25, -math.inf)
        if v > 1:
            x.masked_fill_(rnd(n * v, 1) < 1 / 64, -math.inf)
        s.scores = x.to(dtype)
        s.total = -20.0 * rnd(n, 1) - 3.0 * rnd(n, v).sqrt()
        if v > 1:
            s.total[:, 1:].masked_fill_(rnd(n, v - 1) < 1 / 16, -math.inf)   # (beams that are not there)
        s.done = (rnd(n, v) < case["done"]).to(torch.uint8) if case["done"] > 0 else None
        if own:
            from paper_2302_06126_amd.policy import Beam
            s.call = Beam(n, case["w"], a, width_in=v, dtype=dtype, device=dev)
    elif s.op == "reorder":
        n, w, rows = case["n"], case["w"], case["n"] * case["w"]
        # most beams go on from a few good ones; a beam in 32 has no parent
        s.parent = (rnd(n, w).square() * w).to(torch.int32).clamp_(max=w - 1)
        s.parent.masked_fill_(rnd(n, w) < 1 / 32, -1)
        s.states = [nrm(rows, case["ops"], F_OP), nrm(rows, case["devices"], F_DEV),
                    (rnd(rows, case["ops"] * case["links"]) < 0.3).to(torch.uint8),
                    (rnd(rows, case["depth"]) * 256).to(torch.int32)]
        s.out = s.states if case["place"] else [torch.zeros_like(t) for t in s.states]
        if own:
            from paper_2302_06126_amd.policy import Reorder
            s.call = Reorder(s.states, n, w, out=None if case["place"] else s.out)
    elif s.op == "clip":
        s.g = [(1e-3 * nrm(r, t)).to(torch.bfloat16 if b == 16 else torch.float32)[:, :c] for r, c, t, b in _sizes(case)]
        s.flat, s.out = _flat([(r, c, b) for r, c, _, b in _sizes(case)], dev)
        s.limit = case["limit"] * _norm(s.g)
        if own:
            from paper_2302_06126_amd.optim import Clip
            s.call = Clip(s.g, s.limit, out=s.out)
    else:
        mats, rest = _model_shapes(case["f"], case["layers"], case["hidden"])
        s.w = [nrm(*d) / math.sqrt(d[2]) for d in mats] + [0.1 * nrm(rest)]
        s.g = [_gradient(gen, dev, *d) for d in mats] + [1e-3 * nrm(rest)]
        s.m = [MOMENTUM * _gradient(gen, dev, *d) for d in mats] + [1e-3 * nrm(rest)]
        s.limit = case["limit"] * _norm(s.g)
        if own:
            from paper_2302_06126_amd.optim import Muon
            s.call = Muon(list(zip(s.w, s.g)), lr=LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY,
                          steps=STEPS, coef=COEF, eps=EPS, state=s.m, max_norm=s.limit)
    return s


# --------------------------------------------------------------------------
# the plain form
# --------------------------------------------------------------------------

def _plain_beam(s):
    """In 64 bits: the order of continuations of different beams hangs on their sums."""
    n, v, w, a = (s.case[k] for k in ("n", "v", "w", "s"))
    x = s.scores.double().view(n, v, a)
    top = x.max(dim=2).values
    lse = top + torch.log(torch.exp(x - top[:, :, None]).sum(dim=2))
    c = x + (s.total.double() - lse)[:, :, None]
    c = torch.where((torch.isfinite(s.total) & torch.isfinite(top))[:, :, None], c, -math.inf)
    at = torch.arange(a, device=x.device)
    if s.done is not None:
        done = s.done.bool()
        c = torch.where(done[:, :, None], torch.where(at == 0, s.total.double()[:, :, None], -math.inf), c)
    best, index = torch.sort(c.view(n, v * a), dim=1, descending=True, stable=True)
    k = min(w, v * a)
    total = torch.full((n, w), -math.inf, device=x.device)
    parent = torch.full((n, w), -1, dtype=torch.int32, device=x.device)
    slice_ = parent.clone()
    some = best[:, :k] > -math.inf
    beam = torch.div(index[:, :k], a, rounding_mode="floor")
    total[:, :k] = best[:, :k].float()
    parent[:, :k] = torch.where(some, beam, -1).to(torch.int32)
    keeps = ~some if s.done is None else ~some | torch.gather(done, 1, beam)
    slice_[:, :k] = torch.where(keeps, -1, index[:, :k] % a).to(torch.int32)
    return total, parent, slice_


def _plain_reorder(s):
    n, w = s.parent.shape
    has = (s.parent >= 0).view(-1)
    at = (torch.arange(n, device=has.device)[:, None] * w + s.parent.clamp_min(0)).view(-1)
    for x, y in zip(s.states, s.out):
        rows = x.index_select(0, at)
        y.copy_(torch.where(has.view([-1] + [1] * (x.dim() - 1)), rows, y))
    return s.out


def _plain_scale(g, limit):
    norm = torch.stack([t.double().square().sum() for t in g]).sum().sqrt()
    scale = torch.where(norm > limit, limit / norm, torch.ones_like(norm))
    scale = torch.where(torch.isfinite(norm), scale, torch.zeros_like(norm))
    return norm.float().reshape(1), scale.float()


def _plain_clip(s):
    norm, scale = _plain_scale(s.g, s.limit)
    for g, y in zip(s.g, s.out):
        y.copy_((g.float() * scale).to(g.dtype))
    return s.flat, norm


def _plain_newton_schulz(g):
    x = g.transpose(1, 2) if g.shape[1] > g.shape[2] else g
    x = x / (x.double().square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS).float()
    a, b, c = COEF
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return x.transpose(1, 2) if g.shape[1] > g.shape[2] else x


def _plain_step(s):
    norm, scale = _plain_scale(s.g, s.limit)
    for w, g, m in zip(s.w, s.g, s.m):
        g = g * scale
        m.mul_(MOMENTUM).add_(g)
        u = g + MOMENTUM * m
        w.mul_(1.0 - LR * DECAY)
        if w.dim() == 3:
            u = _plain_newton_schulz(u) * math.sqrt(max(1.0, w.shape[1] / w.shape[2]))
        w.sub_(u, alpha=LR)
    return s.w, s.m, norm


def run(s):
    if own:
        if s.op == "beam":
            return s.call(s.scores, s.total, done=s.done)
        if s.op == "reorder":
            s.call(s.parent)
            return s.out
        if s.op == "clip":
            norm = s.call()
            return s.flat, norm
        s.call.step()
        return s.w, s.m, s.call.norm
    return {"beam": _plain_beam, "reorder": _plain_reorder, "clip": _plain_clip, "step": _plain_step}[s.op](s)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def _ortho_flops(count, rows, cols):
    """The symmetric products take their half."""
    n, m = min(rows, cols), max(rows, cols)
    return float(count) * STEPS * (n * n * m + n * n * n + 2.0 * n * n * m)


def work(case):
    if case["op"] == "beam":
        n, v, w, a = (case[k] for k in ("n", "v", "w", "s"))
        rows = n * v * (1.0 - case["done"])
        return {"bytes": rows * a * (2.0 if case["dtype"] == "bf16" else 4.0) + n * v * 5.0 + n * w * 12.0,
                "flops": 4.0 * rows * a}
    if case["op"] == "reorder":
        n, w = case["n"], case["w"]
        row = 4.0 * (case["ops"] * F_OP + case["devices"] * F_DEV + case["depth"]) + case["ops"] * case["links"]
        # parents w u^2: the share of beams that some beam goes on from; in place a row whose parent it is stays
        read = sum(1.0 - (1.0 - (math.sqrt((p + 1) / w) - math.sqrt(p / w)) * 31 / 32) ** w for p in range(w))
        return {"bytes": n * row * (read + w * 31 / 32) + n * w * 4.0, "flops": 0.0}
    if case["op"] == "clip":
        return {"bytes": sum(r * c * b / 4.0 for r, c, _, b in _sizes(case)) + 4.0,
                "flops": sum(3.0 * r * c for r, c, _, _ in _sizes(case))}
    mats, rest = _model_shapes(case["f"], case["layers"], case["hidden"])
    values = sum(c * r * k for c, r, k in mats) + rest
    return {"bytes": 20.0 * values, "flops": sum(_ortho_flops(*d) for d in mats) + 9.0 * values}


# --------------------------------------------------------------------------
# 64 bits
# --------------------------------------------------------------------------

def _exact_beam(s):
    """Search by search, on the host."""
    n, v, w, a = (s.case[k] for k in ("n", "v", "w", "s"))
    x = s.scores.double().cpu().numpy().reshape(n, v, a)
    before = s.total.double().cpu().numpy()
    done = np.zeros((n, v), bool) if s.done is None else s.done.cpu().numpy().astype(bool)
    total, parent, slice_ = np.full((n, w), -np.inf), np.full((n, w), -1, np.int32), np.full((n, w), -1, np.int32)
    for b in range(n):
        values, beams, slices = [], [], []
        for i in range(v):
            if not np.isfinite(before[b, i]):
                continue
            if done[b, i]:
                values.append([before[b, i]]), beams.append([i]), slices.append([-1])
                continue
            row = x[b, i]
            m = row.max()
            if np.isneginf(m):
                continue
            c = row + (before[b, i] - (m + np.log(np.exp(row - m).sum())))
            keep = np.flatnonzero(c > -np.inf)
            if len(keep) > w:   # (its best, ties among the last of them all kept)
                keep = keep[c[keep] >= np.partition(c[keep], len(keep) - w)[len(keep) - w]]
            values.append(c[keep]), beams.append(np.full(len(keep), i)), slices.append(keep)
        if not values:
            continue
        values, beams, slices = (np.concatenate(p) for p in (values, beams, slices))
        order = np.argsort(-values, kind="stable")[:w]
        total[b, :len(order)], parent[b, :len(order)], slice_[b, :len(order)] = values[order], beams[order], slices[order]
    return total, parent, slice_


def _exact_reorder(s):
    n, w = s.parent.shape
    parent = s.parent.cpu().numpy()
    old = [t.clone() for t in s.states]
    for b in range(n):
        for i in range(w):
            if parent[b, i] >= 0:
                for x, y in zip(old, s.out):
                    y[b * w + i] = x[b * w + parent[b, i]]
    return s.out


def _exact_scale(g, limit):
    total = 0.0
    for t in g:
        total += float((t.double() * t.double()).sum())
    norm = math.sqrt(total)
    return norm, limit / norm if norm > limit else 1.0


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
    if s.op == "beam":
        return _exact_beam(s)
    if s.op == "reorder":
        return _exact_reorder(s)
    norm, scale = _exact_scale(s.g, s.limit)
    if s.op == "clip":
        flat, out = _flat([(r, c, b) for r, c, _, b in _sizes(case)], s.g[0].device, double=True)
        for g, y in zip(s.g, out):
            torch.mul(g.double(), scale, out=y)
        return flat, torch.tensor([norm], dtype=torch.float64)
    ws, ms = [], []
    for w, g, m in zip(s.w, s.g, s.m):
        g = scale * g.double()
        m = MOMENTUM * m.double() + g
        u = g + MOMENTUM * m
        if w.dim() == 3:
            u = math.sqrt(max(1.0, w.shape[1] / w.shape[2])) * _exact_newton_schulz(u)
        ws.append((1.0 - LR * DECAY) * w.double() - LR * u)
        ms.append(m)
    return ws, ms, torch.tensor([norm], dtype=torch.float64)
