"""Plain double-precision CPU statement of the operators around the step: gradient norms and clipping, and gossip by messages in
microscaled 4-bit floating point.  Test infrastructure only; the product never calls it."""

from __future__ import annotations

import numpy as np

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def grad_norm(g, stored):
    """The 2-norm of the stored elements of one gradient."""
    with np.errstate(all="ignore"):
        return np.sqrt(np.sum(np.square(g[stored].astype(np.float64))))


def clip(g, stored, max_norm):
    """(norm, scaled gradient); elements that are not stored stay as they are."""
    n = grad_norm(g, stored)
    out = g.astype(np.float64).copy()
    if not n <= max_norm:
        with np.errstate(all="ignore"):
            out[stored] *= np.float64(max_norm) / n
    return n, out


def message_size(d):
    """(blocks, offset of the scales, bytes)"""
    n = -(-d // BLOCK)
    return n, 16 * n, -(-17 * n // 16) * 16


def encode(x, copy, stored):
    """(message without the bytes that fill it up, values it stands for) of one row: float32 values x, float32 copy or None."""
    d = len(x)
    n, at, _ = message_size(d)
    with np.errstate(all="ignore"):
        u = x.astype(np.float32) - (np.float32(0) if copy is None else copy.astype(np.float32))   # float32 by definition
    u = np.where(stored, u, np.float32(0)).astype(np.float64)
    blocks = np.zeros(n * BLOCK)
    blocks[:d] = u
    blocks = blocks.reshape(n, BLOCK)
    finite = np.isfinite(blocks).all(axis=1)
    a = np.abs(np.where(finite[:, None], blocks, 0.0))
    largest = a.max(axis=1)
    exponent = np.where(largest > 0, np.frexp(largest)[1] - 1, -10000)     # floor(log2)
    exponent = np.maximum(exponent - 2, -126)
    a = a / np.ldexp(1.0, exponent)[:, None]
    code = np.zeros(a.shape, dtype=np.int64)
    for k in range(1, 8):                                                  # past the middle between two magnitudes, or on it to an even code
        middle = (GRID[k] + GRID[k - 1]) / 2
        code[(a > middle) | ((a == middle) & (k % 2 == 0))] = k
    values = GRID[code] * np.ldexp(1.0, exponent)[:, None] * np.where(np.signbit(blocks), -1.0, 1.0)
    values[~finite] = np.nan
    code = np.where(finite[:, None], code + 8 * np.signbit(blocks), 0).reshape(-1)
    scale = np.where(finite, exponent + 127, 255)
    message = np.concatenate([code[0::2] + 16 * code[1::2], scale]).astype(np.uint8)
    return message, values.reshape(-1)[:d]


def decode(message, d):
    n, at, _ = message_size(d)
    codes = np.asarray(message[:at]).astype(np.int64)
    nibble = np.stack([codes & 15, codes >> 4], axis=1).reshape(-1)
    scale = np.asarray(message[at:at + n]).astype(np.float64)
    power = np.where(scale == 255, np.nan, np.exp2(scale - 127))
    return (GRID[nibble & 7] * np.where(nibble & 8, -1.0, 1.0) * np.repeat(power, BLOCK))[:d]


def product(messages, row_ptr, col, w, d):
    """(W times the messages' values, the same of magnitudes), row by row."""
    got, size = [], []
    values = {int(c): decode(messages[int(c)], d) for c in set(int(c) for c in col)}
    for i in range(len(row_ptr) - 1):
        terms = [float(np.float32(w[k])) * values[int(col[k])] for k in range(row_ptr[i], row_ptr[i + 1])]
        got.append(np.sum(terms, axis=0))
        size.append(np.sum(np.abs(terms), axis=0))
    return got, size


def gossip(messages, total, copy, x, row_ptr, col, w, gamma):
    """(sums, x behind) of every row, from float32 or bfloat16 values widened."""
    mixed, _ = product(messages, row_ptr, col, w, len(x[0]))
    total = [s.astype(np.float64) + m for s, m in zip(total, mixed)]
    return total, [v.astype(np.float64) + float(np.float32(gamma)) * (s - c) for v, s, c in zip(x, total, copy)]
