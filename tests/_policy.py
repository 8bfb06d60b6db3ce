"""Plain restatements of the operators on scores, for their tests: y of the
constrained priors in the header's own order of fp32 operations (so that the
argmax and the constrained scores have one right answer), everything else in
64 bits."""
import numpy as np

EPS = 2.0 ** -24    # half a step of fp32, relative


def constrained(x, allow=None, bias=None, history=None, lens=None, rep=None, pre=None, frq=None):
    """y [Q, S] fp32 and the largest magnitude that any step of it had."""
    y = np.array(x, np.float32)
    Q, S = y.shape
    top = np.abs(np.where(np.isfinite(y), y, 0)).max(initial=0.0)
    one = np.ones(Q, np.float32)
    rep, pre, frq = (one if rep is None else rep), (0 * one if pre is None else pre), (0 * one if frq is None else frq)
    with np.errstate(all="ignore"):
        if history is not None:
            history = np.broadcast_to(history, (Q, history.shape[-1]))
            for q in range(Q):
                n = history.shape[1] if lens is None else int(np.clip(lens[q], 0, history.shape[1]))
                h = history[q, :n]
                a, c = np.unique(h[(h >= 0) & (h < S)], return_counts=True)
                v = y[q, a]
                v = np.where(v > 0, v / rep[q], v * rep[q])
                v = v - frq[q] * c.astype(np.float32)
                y[q, a] = v - pre[q]
                top = max(top, np.abs(v[np.isfinite(v)]).max(initial=0.0))
        if bias is not None:
            y = y + np.broadcast_to(bias, y.shape)
            top = max(top, np.abs(np.where(np.isfinite(y), y, 0)).max(initial=0.0))
        if allow is not None:
            words = np.ascontiguousarray(allow).view(np.uint32)
            bits = (words[..., np.arange(S) // 32] >> (np.arange(S) % 32).astype(np.uint32)) & 1
            y = np.where(np.broadcast_to(bits, y.shape) != 0, y, -np.inf)
    return y.astype(np.float32), float(top)


def priors(y):
    """(prior in 64 bits, argmax, best) of constrained scores."""
    y = np.asarray(y, np.float64)
    nan = np.isnan(y).any(axis=1)
    best = np.where(np.isnan(y), -np.inf, y).max(axis=1)
    none = np.isneginf(best)
    with np.errstate(invalid="ignore"):
        e = np.exp(y - np.where(none, 0.0, best)[:, None])
        p = e / np.where(none, 1.0, e.sum(axis=1))[:, None]
    p[nan] = np.nan
    at = np.where(np.isnan(y), -np.inf, y).argmax(axis=1)
    return p, np.where(nan | none, -1, at).astype(np.int32), np.where(nan, np.nan, best)


def shares(masks, n_dev):
    bits = ((np.asarray(masks, np.uint64)[:, None] >> np.arange(n_dev, dtype=np.uint64)) & np.uint64(1)).astype(np.float64)
    return bits / np.maximum(bits.sum(axis=1, keepdims=True), 1.0)


def balance_loss(x, masks, n_dev, coef, use, load):
    """The loss with the load held (what its gradient is of)."""
    use = np.asarray(use, bool) & ~np.isneginf(x).all(axis=1)
    n = use.sum()
    if n == 0:
        return 0.0
    e = np.exp(x[use] - x[use].max(axis=1, keepdims=True))
    p = e / e.sum(axis=1, keepdims=True)
    return coef * n_dev * float((p.mean(axis=0) @ shares(masks, n_dev)) @ load)


def balance(x, masks, n_dev, coef, use=None):
    """(loss, grad, count, load, h) in 64 bits."""
    x = np.asarray(x, np.float64)
    Q, S = x.shape
    use = (np.ones(Q, bool) if use is None else np.asarray(use, bool)) & ~np.isneginf(x).all(axis=1)
    n, A = int(use.sum()), shares(masks, n_dev)
    count = np.bincount(x[use].argmax(axis=1), minlength=S).astype(np.int32) if n else np.zeros(S, np.int32)
    load = count @ A / max(n, 1)
    h = A @ load
    grad = np.zeros_like(x)
    if n:
        e = np.exp(x[use] - x[use].max(axis=1, keepdims=True))
        p = e / e.sum(axis=1, keepdims=True)
        grad[use] = coef * n_dev / n * p * (h - (p @ h)[:, None])
    return balance_loss(x, masks, n_dev, coef, use, load), grad, count, load, h
