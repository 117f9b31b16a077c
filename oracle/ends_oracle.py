"""Plain 64-bit statements of the operators at the ends of an iteration: the Newton-Schulz iteration that orthogonalises a matrix, the step along
it, and the loss of a head with its gradients.  Test infrastructure only."""

import numpy as np

SCHEDULE = [(3.4445, -4.7750, 2.0315)] * 5


def orthogonalised(m, schedule=SCHEDULE):
    """X = M / (|M| + 1e-7), then X = a X + (b A + c A A) X with A = X X^T, of the transpose if the matrix is tall."""
    m = np.asarray(m, dtype=np.float64)
    x = m.T if m.shape[0] > m.shape[1] else m
    x = x / (np.sqrt((x * x).sum()) + 1e-7)
    for a, b, c in schedule:
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if m.shape[0] > m.shape[1] else x


def orthogonalised_error(m, planes, schedule=SCHEDULE):
    """A bound of the 2-norm of what the library's roundings make of orthogonalised(m).

    Operands carry 11 bits a plane: half a step is u1 = 2^-11 of an element with one plane and 2^-22 with two; X is held to 2^-22 in any case.  A sum of K
    products in float32 is off by about sqrt(K) roundings of 2^-24 of the magnitudes' sum, four times that is taken.  What one iteration is off, the next
    multiplies by at most the largest derivative of its polynomial on the singular values."""
    x = np.asarray(m, dtype=np.float64)
    x = x.T if x.shape[0] > x.shape[1] else x
    x = x / (np.sqrt((x * x).sum()) + 1e-7)
    u1, u2 = 2.0 ** -11 if planes == 1 else 2.0 ** -22, 2.0 ** -22
    f = np.linalg.norm
    sums = lambda k: 4 * np.sqrt(k) * 2.0 ** -24  # noqa: E731
    e = 2.0 ** -23 * f(x)
    for a, b, c in schedule:
        g = x @ x.T
        gg = g @ g
        B = b * g + c * gg
        top = np.linalg.norm(x, 2) if min(x.shape) else 0.0
        t = np.linspace(0, max(1.0, 1.05 * top), 400)
        slope = np.abs(a + 3 * b * t ** 2 + 5 * c * t ** 4).max()
        dg = 2 * u1 * top * f(x) + sums(x.shape[1]) * f(np.abs(x) @ np.abs(x).T) + u1 * f(g)
        dgg = 2 * top ** 2 * (dg + u1 * f(g)) + sums(len(g)) * f(np.abs(g) @ np.abs(g))
        db = abs(b) * dg + abs(c) * dgg + 2.0 ** -23 * f(B) + u1 * f(B)
        e = slope * (e + u2 * f(x)) + top * db + f(B, 2) * u1 * f(x) + sums(len(g)) * f(np.abs(B) @ np.abs(x)) + 2.0 ** -23 * f(a * x)
        x = a * x + B @ x
    return e + 2.0 ** -22 * f(x)
