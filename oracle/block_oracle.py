"""Plain definitions in 64 bits of what lies between the attention calls of a block: counter-based dropout and layer
norm with the residual sum and the dropout in front of it."""
import numpy as np


def philox4x32(counter, key, rounds=10):
    """Philox-4x32 (Salmon, Moraes, Dror, Shaw, SC 2011) in Python integers: four words of counter, two of key."""
    a, b, c, d = (int(x) for x in counter)
    k0, k1 = (int(x) for x in key)
    for _ in range(rounds):
        p, q = 0xD2511F53 * a, 0xCD9E8D57 * c
        a, b, c, d = (q >> 32) ^ b ^ k0, q & 0xFFFFFFFF, (p >> 32) ^ d ^ k1, p & 0xFFFFFFFF
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return a, b, c, d


def threshold(p):
    """Of 65536 equally likely half words, how many drop the value."""
    return min(65535, int(np.floor(65536.0 * float(np.float32(p)) + 0.5)))


def keep_mask(rows, cols, seed, offset, site, p):
    """Factors of the values, [rows, cols] float64: 0 or 65536 / (65536 - t)."""
    t, out = threshold(p), np.zeros((rows, cols))
    key = (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF)
    for r in range(rows):
        for c0 in range(0, cols, 8):
            words = philox4x32((c0 // 8, r, site & 0xFFFFFFFF, offset & 0xFFFFFFFF), key)
            for c in range(c0, min(c0 + 8, cols)):
                half = words[(c - c0) // 2] >> (16 * ((c - c0) % 2)) & 0xFFFF
                out[r, c] = 65536.0 / (65536 - t) if half >= t else 0.0
    return out


def layer_norm(h, weight, bias, eps):
    """(y, mean, rstd)."""
    mean = h.mean(1)
    rstd = 1.0 / np.sqrt(((h - mean[:, None]) ** 2).mean(1) + eps)
    return (h - mean[:, None]) * rstd[:, None] * weight + bias, mean, rstd


def layer_norm_bwd(d_y, h, mean, rstd, weight, d_h=None):
    """(d_residual, d_weight, d_bias)."""
    xhat = (h - mean[:, None]) * rstd[:, None]
    g = d_y * weight
    d = rstd[:, None] * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    return (d if d_h is None else d + d_h), (d_y * xhat).sum(0), d_y.sum(0)
