"""Plain 64-bit forms of what stands between the layers of a residual block: dropout from a counter-based generator, the residual's
addition with a root-mean-square norm and their gradients, rows and weights in 8 bits, and layers that multiply them.  Untiled."""
from fractions import Fraction

import numpy as np


def philox(counter, key, rounds=10):
    """Philox4x32 of four counter words under two key words, in Python's whole numbers"""
    x, k = [int(v) for v in counter], [int(v) for v in key]
    for _ in range(rounds):
        a, b = 0xD2511F53 * x[0], 0xCD9E8D57 * x[2]
        x = [(b >> 32) ^ x[1] ^ k[0], b & 0xffffffff, (a >> 32) ^ x[3] ^ k[1], a & 0xffffffff]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return x


def dropped_below(p):
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def keep_mask(rows, cols, p, seed, offset):
    """True where a value is kept"""
    below = dropped_below(p)
    keep = np.zeros((rows, cols), dtype=bool)
    offset %= 1 << 64
    for r in range(rows):
        for c in range(cols):
            if c % 8 == 0:
                w = philox((c // 8, r, offset & 0xffffffff, offset >> 32), (seed & 0xffffffff, seed >> 32 & 0xffffffff))
            keep[r, c] = (w[c % 8 // 2] >> 16 * (c % 2) & 0xffff) >= below
    return keep


def dropout(X, p, keep):
    """X where it is kept, by the probability that is applied; 0 elsewhere whatever X holds"""
    return np.where(keep, np.where(keep, X, 0.0) * (65536.0 / (65536 - dropped_below(p))), 0.0)


def norm(H, gain, eps):
    """(Y, 1 / root mean square)"""
    r = 1.0 / np.sqrt(np.mean(H * H, axis=1, keepdims=True) + eps)
    return H * r * gain, r


def norm_backward(H, gain, eps, dY, dH):
    """(gradient of the sum, of the gain)"""
    _, r = norm(H, gain, eps)
    n = H * r
    c = np.mean(gain * dY * n, axis=1, keepdims=True)
    return r * (gain * dY - c * n) + dH, np.sum(dY * n, axis=0)


def nearest_step(u, m):
    """127 u / m to the nearest whole number, ties to even, in fractions"""
    return round(Fraction(127) * Fraction(float(u)) / Fraction(float(m)))


def steps(U):
    """(Q, largest magnitudes) of the rows of U (exact 64-bit values); rows that hold something that is not a number: Q = 0, NaN"""
    Q, most = np.zeros(U.shape, dtype=np.int64), np.zeros(U.shape[0])
    for t, u in enumerate(U):
        most[t] = np.max(np.abs(u)) if len(u) and np.all(np.isfinite(u)) else np.nan if len(u) else 0.0
        if not most[t] > 0:
            continue
        x = 127.0 * (u / most[t])
        q = np.rint(x)
        for i in np.nonzero(np.abs(np.abs(x - q) - 0.5) < 1e-9)[0]:
            q[i] = nearest_step(u[i], most[t])
        Q[t] = q
    return Q, most


def layer8(XQ, XS, WQ, WS, relu):
    """XQ: tokens x inputs, WQ: inputs x outputs, whole numbers; scales in 64 bits"""
    total = XQ.astype(np.float64) @ WQ.astype(np.float64)      # (whole numbers below 2^53: exact in any order)
    Y = total * WS[None, :] * XS[:, None]
    return np.where(Y < 0, 0.0, Y) if relu else Y
