"""Double-precision definitions of the orthogonalised update in numpy, turn by turn.  Test infrastructure; shares no code with the CUDA
path."""
import numpy as np

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def iterates(x, steps, coefficients=COEFFICIENTS, eps=1e-7):
    """X_0, X_1, ... of one matrix, over its shorter side."""
    a, b, c = coefficients
    x = x.astype(np.float64)
    x = x / (np.sqrt((x ** 2).sum()) + eps)
    out = [x]
    for _ in range(steps):
        x = out[-1]
        if x.shape[0] <= x.shape[1]:
            g = x @ x.T
            out.append(a * x + (b * g + c * g @ g) @ x)
        else:
            g = x.T @ x
            out.append(a * x + x @ (b * g + c * g @ g))
    return out


def by_singular_values(x, steps, coefficients=COEFFICIENTS, eps=1e-7):
    """The same from the singular value decomposition."""
    a, b, c = coefficients
    u, s, v = np.linalg.svd(x.astype(np.float64), full_matrices=False)
    s = s / (np.sqrt((s ** 2).sum()) + eps)
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return (u * s) @ v


def tolerance(its, coefficients=COEFFICIENTS):
    """Frobenius norm of the error that pieces of 22 bits and 32-bit sums may leave, given the iterates in 64 bits.

    A turn stores X, A and P (2^-22 of each value), leaves out lo lo (2^-22 of a product) and adds K values in groups of 16 that a sum may
    cut off rather than round (2^-23 of the sum each; A: K / 16 groups over two sums of a block, so K / 32 of them for a sum of all; P X: at
    most K / 16; together under K / 10): d = 5 * 2^-22 + (K / 10 + 4) * 2^-23 of |a| |X| + |b| |X|^3 + |c| |X|^5 with |X| <= 1.3, less than 14 times the Frobenius norm of X.  A later turn stretches an error at most by the
    largest derivative of a v + b v^3 + c v^5, max(|a|, ...) over the values met, 5 here."""
    a, b, c = coefficients
    k = max(its[0].shape)
    d = 5 * 2.0 ** -22 + (k / 10 + 4) * 2.0 ** -23
    grow = max(abs(a + 3 * b * v ** 2 + 5 * c * v ** 4) for v in np.linspace(0, 1.25, 100))
    total = 0.0
    for x in its[:-1]:
        total = grow * total + 14 * d * np.sqrt((x ** 2).sum())
    return total


def in_32_bits(x, steps, coefficients=COEFFICIENTS, eps=1e-7):
    """The last iterate by products of 32-bit numbers."""
    if x.shape[0] > x.shape[1]:
        return in_32_bits(x.T, steps, coefficients, eps).T
    a, b, c = (np.float32(v) for v in coefficients)
    x = x.astype(np.float32)
    x = x / (np.sqrt((x ** 2).sum()) + np.float32(eps))
    for _ in range(steps):
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.astype(np.float64)


def near(err32, k):
    """Relative Frobenius norm of the error that may be left where the same turns in 32-bit products leave err32 on the same matrix; k is
    its longer side.

    What 32 bits round by 2^-24 is rounded by 2^-23 as two pieces, for both operands of a product, and lo lo (2^-24 of it) is left out: less than
    four times the rounding errors, wherever they are made and however they grow.  Sums that are cut off rather than rounded lose 2^-24 of themselves
    on average, K / 32 times, at most 128 times before they are added up elsewhere, and P's derivative with respect to A is at most 2 in
    effect: 2^-28 for each K up to 4096.  2^-21 stands for an err32 that happens to be small."""
    return 4 * err32 + min(k, 4096) * 2.0 ** -28 + 2.0 ** -21
