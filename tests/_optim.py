"""The Newton-Schulz iteration in 64 bits, and how far the kernels may be from it.

Products of two-part fp16 splits: an operand is held to 2^-22 of itself, what a
product leaves out is below 2^-22 of it, and the fp32 sum of 3 K / 16 partial
results is rounded (towards minus infinity, half of the terms negated) by at
most 2^-23 of a partial sum each, errors that add up like their root.  With
||B|| <= 3 and ||A|| <= 1.5 (the quintic; others stay below 15) a step's own
error, relative to the ||X||_F that it leaves, is at most
  e = 3 (2^-22 * 4 + 2^-23 * sqrt(3 K / 16)) * 3
(three products, each of operands below 3), and a step multiplies an error that
it is given by at most L = max |p'| = 4 over the singular values' range, so

  ||error||_F <= sum_k L^(steps - 1 - k) e ||X_{k+1}||_F .

Elements: 10 root-mean-squares of that, for up to 2^23 of them.  The bf16 form
multiplies operands rounded to fp16 (2^-11 in place of 2^-22) but carries X to
2^-22: an operand's rounding error reaches X through B X alone, along singular
directions that B has already raised, and is not raised again (L = 1); the
result is rounded by at most 2^-8 of each element."""
import numpy as np

QUINTIC = (3.4445, -4.7750, 2.0315)


def newton_schulz(g, steps=5, coef=QUINTIC, eps=1e-7):
    """(result, the X of every step) in 64 bits, by singular values."""
    g = np.asarray(g, np.float64)
    u, s, vt = np.linalg.svd(g, full_matrices=False)
    s = s / (np.sqrt((g * g).sum()) + eps)
    a, b, c = coef
    norms = [np.sqrt((s * s).sum())]
    for _ in range(steps):
        s = s * (a + b * s ** 2 + c * s ** 4)
        norms.append(np.sqrt((s * s).sum()))
    return (u * s) @ vt, norms


def tolerance(shape, norms, steps=5, bf16=False):
    """(of the Frobenius norm, of an element less its own rounding)."""
    K = max(64, -(-max(shape) // 64) * 64)
    held = 2.0 ** -11 if bf16 else 2.0 ** -22
    e = 9 * (4 * held + 2.0 ** -23 * np.sqrt(3 * K / 16))
    L = 1.0 if bf16 else 4.0
    total = sum(L ** (steps - 1 - k) * e * norms[k + 1] for k in range(steps))
    if bf16:   # X's own error is raised all the same
        total += sum(4.0 ** (steps - 1 - k) * 9 * 2.0 ** -20 * norms[k + 1] for k in range(steps))
    return total, 10 * total / np.sqrt(min(shape) * max(shape))


def rounded_bf16(g, steps=5, coef=QUINTIC, eps=1e-7):
    """The iteration of products in 64 bits with the operands' roundings of the
    bf16 form: 2^12 times X, A and B in fp16, the diagonals of A and B apart
    from them and exact, X held in two parts."""
    def held(x, parts):
        x = 4096.0 * x
        hi = x.astype(np.float16).astype(np.float64)
        return (hi + (0.0 if parts == 1 else (x - hi).astype(np.float16).astype(np.float64))) / 4096.0

    g = np.asarray(g, np.float64)
    x = g if g.shape[0] <= g.shape[1] else g.T
    x = held(x / (np.sqrt((x * x).sum()) + eps), 2)
    a, b, c = coef
    eye = np.eye(x.shape[0])
    for _ in range(steps):
        xh = held(x, 1)
        A = xh @ xh.T
        d = np.diag(A)
        off = A - eye * d
        offh = held(off, 1)
        B = b * A + c * (offh @ offh + (d[:, None] + d[None]) * held(off, 2) + eye * (d * d))
        e = np.diag(B)
        x = held(a * x + e[:, None] * xh + held(B - eye * e, 1) @ xh, 2)
    return x if g.shape[0] <= g.shape[1] else x.T
