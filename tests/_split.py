"""The Newton-Schulz iteration with every rounding of the kernels' products, on
the CPU: operands of 2^12 times their value in two fp16 parts, products of
hi hi', hi lo' and lo hi' summed in fp32 by fragments of 16 k (even and odd ones
apart, the odd ones negated), each partial sum rounded towards minus infinity as
the matrix cores do, the terms around the products in fp32.

BOUND is what fp32 results may be off by, relative to their Frobenius norm, for
five steps of the quintic and matrices of up to about 2,000 columns.  The
iteration below is off by at most 7.5e-6 up to 400 x 400 and 300 x 900 (3e-6 at
the shapes of test_optim_split.py).  Its errors are independent roundings, whose
share of the norm does not grow with the matrix, but for those of the sums, which
grow with the root of K / 16: from 57 fragments there to 132, by 1.5.  2^-15
leaves sums in another order 2.7 times that, and is a sixteenth of what a missing
cross product costs (5e-4 and more).
"""
import numpy as np

from tests import _optim as R

BOUND = 2.0 ** -15


def _parts(x):
    hi = x.astype(np.float16)
    return hi.astype(np.float64), (x - hi.astype(np.float32)).astype(np.float16).astype(np.float64)


def _down(x):
    """fp32, towards minus infinity."""
    f = x.astype(np.float32)
    return np.where(f.astype(np.float64) > x, np.nextafter(f, np.float32(-np.inf)), f)


def _product(r, s, keep):
    """r s^T of matrices in two parts, times 2^-12."""
    k = r[0].shape[1]
    sums = [np.zeros((r[0].shape[0], s[0].shape[0]), np.float32) for _ in range(2)]
    for f, at in enumerate(range(0, k, 16)):
        sign = -1.0 if f % 2 else 1.0
        for i, (p, q) in enumerate(((1, 0), (0, 1), (0, 0))):
            if i in keep:
                sums[f % 2] = _down(sums[f % 2].astype(np.float64) + sign * r[p][:, at:at + 16] @ s[q][:, at:at + 16].T)
    return (sums[0] - sums[1]) * np.float32(2.0 ** -12)


def iterate(g, steps=5, coef=R.QUINTIC, eps=1e-7, keep=(0, 1, 2)):
    """keep: which of lo hi', hi lo', hi hi' a product adds."""
    g = np.asarray(g, np.float32)
    x = g if g.shape[0] <= g.shape[1] else g.T
    d = x.astype(np.float64)
    x = (d * (4096.0 / (np.sqrt((d * d).sum()) + eps))).astype(np.float32)
    a, b, c = (np.float32(v) for v in coef)
    own = lambda p: (p[0] + p[1]).astype(np.float32)
    for _ in range(steps):
        p = _parts(x)
        A = _parts(_product(p, p, keep))
        B = _parts(b * own(A) + c * _product(A, A, keep))
        x = a * own(p) + _product(B, [v.T for v in p], keep)
    x = x.astype(np.float64) / 4096.0
    return x if g.shape[0] <= g.shape[1] else x.T
