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


def _halves(v):
    """(high, low): 11 bits each of float32 values, of whatever size."""
    fraction, exponent = np.frexp(v.astype(np.float64))
    high = np.ldexp(np.rint(fraction * 2048) / 2048, exponent).astype(np.float32)
    fraction, exponent = np.frexp(v.astype(np.float64) - high)
    return high, np.ldexp(np.rint(fraction * 2048) / 2048, exponent).astype(np.float32)


def orthogonalised_with_roundings(m, planes, schedule=SCHEDULE):
    """orthogonalised(m) with the operands' bits that the library states: X in two halves, A and B in one half (planes 1) or two, B's diagonal apart in float32; products
    of one half a side or of two without low times low, sums in float32."""
    m = np.asarray(m, dtype=np.float64)
    x = m.T if m.shape[0] > m.shape[1] else m
    x = x.astype(np.float32) * np.float32(1 / (np.sqrt((x * x).sum()) + 1e-7))

    def product(p, q):
        return p[0] @ q[0] + (p[0] @ q[1] + p[1] @ q[0]) if planes == 2 else p[0] @ q[0]

    for a, b, c in np.asarray(schedule, dtype=np.float32):
        h = _halves(x)
        g = _halves(product(h, (h[0].T, h[1].T)))
        B = b * (g[0] + g[1] if planes == 2 else g[0]) + c * product(g, g)
        diagonal = np.diag(B).copy()
        np.fill_diagonal(B, 0)
        x = (h[0] + h[1]) * (a + diagonal)[:, None] + product(_halves(B), h)
    return x.T if m.shape[0] > m.shape[1] else x


def orthogonalised_spread(m, planes, schedule=SCHEDULE, draws=4, seed=0):
    """How far (2-norm) the roundings of orthogonalised_with_roundings take the result, at most, over m and copies of it whose elements differ in their last places: the
    library's sums are in another order, which leaves roundings as large but turns some the other way."""
    rng, m = np.random.default_rng(seed), np.asarray(m, dtype=np.float64)
    want, most = orthogonalised(m, schedule), 0.0
    for k in range(draws):
        near = m if k == 0 else m * (1 + rng.uniform(-1, 1, m.shape) * 2.0 ** -22)
        most = max(most, np.linalg.norm(orthogonalised_with_roundings(near, planes, schedule) - want))
    return most


def orthogonalised_error_of_a_row(m, planes, schedule=SCHEDULE):
    """A bound like orthogonalised_error's for a matrix of one row or column, whose roundings are too few to say anything about another draw of them.

    X is s times a unit vector, so A = s^2 and B, all diagonal, are numbers.  An operand is off by u = 2^-22 of itself, or of the products' 2^-11 with one plane; a sum of K
    products by 4 sqrt(K) roundings of 2^-24.  A is off by 2 u A and its sum, and by u A as it is held; B = b A + c A A by |b + 2 c A| times that, the product's sum and two roundings; a X +
    B X by u of X, by s times what B is off and by three roundings.  What X is off already grows by the polynomial's slope along X and by p(s) / s across it."""
    s = np.linalg.norm(np.asarray(m, dtype=np.float64))
    s, size = s / (s + 1e-7), np.asarray(m).size
    u, e = 2.0 ** -11 if planes == 1 else 2.0 ** -22, 2.0 ** -23
    for a, b, c in schedule:
        A = s * s
        B = b * A + c * A * A
        dA = (3 * u + 4 * np.sqrt(size) * 2.0 ** -24) * A
        dB = abs(b + 2 * c * A) * dA + abs(c) * (dA * dA + 4 * 2.0 ** -24 * A * A) + 2.0 ** -23 * (abs(b) * A + abs(c) * A * A)
        local = 2.0 ** -22 * s * abs(a + B) + s * dB + 3 * 2.0 ** -24 * s * (abs(a) + abs(B))
        e = max(abs(a + 3 * b * A + 5 * c * A * A), abs(a + B)) * e + local
        s = s * abs(a + B)
    return 1.01 * e


def head_loss(hidden, head, bias, targets, scale=1.0, mean=True):
    """{"loss", "nll", "dz", "dhidden", "dhead", "dbias"} of one replica; tokens without a target take no part."""
    with np.errstate(invalid="ignore", over="ignore"):
        w, y = np.asarray(head, dtype=np.float64), np.asarray(targets)
        taken = (y >= 0) & (y < len(w))
        h = np.where(taken[:, None], np.asarray(hidden, dtype=np.float64), 0.0)
        z = h @ w.T + (0 if bias is None else np.asarray(bias, dtype=np.float64))
        top = z.max(axis=1, keepdims=True) if len(z) else z
        lse = (top + np.log(np.exp(z - top).sum(axis=1, keepdims=True)))[:, 0] if len(z) else np.zeros(0)
        s = scale / (max(1, int(taken.sum())) if mean else 1)
        word = np.where(taken, y, 0)
        nll = np.where(taken, lse - z[np.arange(len(y)), word], 0.0)
        dz = np.exp(z - lse[:, None])
        dz[np.arange(len(y)), word] -= 1
        dz = np.where(taken[:, None], dz, 0.0)
        return {"loss": s * nll.sum(), "nll": nll, "dz": dz, "s": s, "z": z, "h": h, "dhidden": s * dz @ w, "dhead": s * dz.T @ h, "dbias": s * dz.sum(axis=0)}


def head_loss_error(r, head, bias, planes, half):
    """Bounds, element by element, of what the library's roundings make of head_loss's results r.  half: half a step of the results' type.

    Logits: operands of 2^-22 a plane pair (of one bfloat16 plane: as given), a sum of K products in float32 off by four times sqrt(K) roundings of 2^-24.
    softmax: twice a logit's error, an exponential good to 2^-21 and to 2^-23 of its argument; held to 2^-22 twice and 2^-38 of 1, or to
    2^-11 and 2^-40 of the largest and then to 2^-8 (half precision, then bfloat16: (1 + 2^-11) (1 + 2^-8) - 1 < 2^-8 + 2^-10).
    What is below 2^-126, float32's (and bfloat16's) smallest normal number, may come out as 0: an exponential of -100 is 2^-144, off by all of itself."""
    w = np.abs(np.asarray(head, dtype=np.float64))
    h, z, s = np.abs(r["h"]), r["z"], abs(r["s"])
    sums = lambda k: 4 * np.sqrt(max(1, k)) * 2.0 ** -24  # noqa: E731
    operand = 2.0 ** -21 if planes == 2 else 0.0
    dlogit = (operand + sums(w.shape[1])) * (h @ w.T) + 2.0 ** -38 * planes * (h.sum(1)[:, None] * w.max(initial=0) + w.sum(1)[None] * h.max(initial=0))
    if bias is not None:
        dlogit = dlogit + 2.0 ** -23 * np.abs(np.where(np.isfinite(z), z, 0))
    worst = dlogit.max(axis=1) if len(z) else np.zeros(0)
    taken = (r["dz"] != 0).any(axis=1)
    finite = np.where(np.isfinite(z), np.abs(z), 0)
    nll = np.where(taken | (r["nll"] != 0), 2 * worst + 2.0 ** -20 + 2.0 ** -22 * (finite.max(axis=1) if len(z) else 0) + 2.0 ** -22 * np.abs(r["nll"]), 0.0)
    dz = np.abs(r["dz"])
    p = np.where(r["dz"] < 0, 1 + r["dz"], r["dz"])
    relative = 2 * worst[:, None] + 2.0 ** -20 + 2.0 ** -22 * finite
    held = (2.0 ** -21 * dz + 2.0 ** -38) if planes == 2 else (2.0 ** -8 + 2.0 ** -10) * dz + 2.0 ** -40
    ddz = np.where(taken[:, None], relative * (p + dz) + held + 2.0 ** -126, 0.0)
    k, t = w.shape[0], len(z)
    lost = 2.0 ** -126
    tiny = 2.0 ** -38 * planes
    return {"nll": nll, "loss": s * nll.sum() + 2.0 ** -23 * abs(r["loss"]),
            "dhidden": s * (ddz @ w + (operand + sums(k) + 2.0 ** -22) * (dz @ w) + tiny * dz.sum(1)[:, None] * w.max(initial=0)) + half * np.abs(r["dhidden"]) + lost,
            "dhead": s * (ddz.T @ h + (operand + sums(t) + 2.0 ** -22) * (dz.T @ h) + tiny * dz.sum(0)[:, None] * h.max(initial=0)) + half * np.abs(r["dhead"]) + lost,
            "dbias": s * (ddz.sum(axis=0) + (sums(t) + 2.0 ** -22) * dz.sum(axis=0)) + half * np.abs(r["dbias"]) + lost}
