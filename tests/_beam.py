"""Plain restatement in 64 bits of a level of beam search (include/tag_beam.h)
and of the reordering of states, one search and one beam after the other."""
import numpy as np

HALF = 2.0 ** -24   # half a step of fp32, relative


def offsets(x, total, done):
    """Per beam: what is added to its scores (-inf: it has no candidates)."""
    x, total = np.asarray(x, np.float64), np.asarray(total, np.float64)
    off = np.full(len(x), -np.inf)
    for v in range(len(x)):
        if not np.isfinite(total[v]):
            continue
        if done[v]:
            off[v] = total[v]
            continue
        m = x[v].max() if not np.isnan(x[v]).any() else np.nan
        if np.isfinite(m):
            off[v] = total[v] - (m + np.log(np.exp(x[v] - m).sum()))
    return off


def select(x, total, done, width):
    """x [n, V, S], total [n, V], done [n, V] -> total (64 bits), parent, slice
    [n, width], and per search how far apart neighbouring ones of the best
    width + 1 candidates are where they differ and belong to different beams."""
    n, V, S = x.shape
    out = np.full((n, width), -np.inf)
    parent = np.full((n, width), -1, np.int32)
    slice_ = np.full((n, width), -1, np.int32)
    gap = np.full(n, np.inf)
    for b in range(n):
        off = offsets(x[b], total[b], done[b])
        key, idx = [], []
        for v in range(V):
            if off[v] == -np.inf:
                continue
            if done[b, v]:
                key.append([off[v]])
                idx.append([v * S])
                continue
            c = np.asarray(x[b, v], np.float64) + off[v]
            a = np.flatnonzero(c > -np.inf)
            key.append(c[a])
            idx.append(v * S + a)
        if not key:
            continue
        key, idx = np.concatenate(key), np.concatenate(idx)
        order = np.lexsort((idx, -key))[:width + 1]
        k, v = key[order], idx[order] // S
        d = (k[:-1] - k[1:])[v[:-1] != v[1:]]
        if (d > 0).any():
            gap[b] = d[d > 0].min()
        order = order[:width]
        out[b, :len(order)] = key[order]
        parent[b, :len(order)] = idx[order] // S
        slice_[b, :len(order)] = np.where(done[b, idx[order] // S], -1, idx[order] % S)
    return out, parent, slice_, gap


def noise(x, total):
    """Bound on what rounding in 64 bits does to a candidate: S positive terms of
    two roundings each and as many additions, and four of the sum's parts."""
    f = np.abs(np.where(np.isfinite(x), x, 0.0)).max(initial=0.0)
    t = np.abs(np.where(np.isfinite(total), total, 0.0)).max(initial=0.0)
    return 2.0 ** -53 * (x.shape[-1] + 4 + 4 * (2 * f + t + np.log(x.shape[-1])))


def check(got, x, total, done, width):
    """got: (total, parent, slice) as arrays.  Parents and slices are exact: where
    neighbours are further apart than the noise, or the same to the bit (one beam,
    or beams that are copies of one another), the order has one right answer."""
    want, parent, slice_, gap = select(x, total, done, width)
    eps = noise(np.asarray(x, np.float64), np.asarray(total, np.float64))
    assert gap.min(initial=np.inf) > 2 * eps, "inputs whose order is not determined"
    assert np.array_equal(got[1], parent)
    assert np.array_equal(got[2], slice_)
    assert np.array_equal(np.isneginf(got[0]), np.isneginf(want))
    ok = np.isfinite(want)
    err = np.abs(got[0].astype(np.float64)[ok] - want[ok])
    assert np.all(err <= HALF * np.abs(want[ok]) + eps + 2.0 ** -149), float(err.max())


def reorder(old, out, parent, width_in):
    """old [n, V, ...] and out [n, W, ...] (what stood there) -> out."""
    out = out.copy()
    n, W = parent.shape
    for b in range(n):
        for w in range(W):
            if 0 <= parent[b, w] < width_in:
                out[b, w] = old[b, parent[b, w]]
    return out
