"""The linear layer, activations and 8-bit checkpoints in 64 bits (numpy), written from their formulas, and what an
implementation in binary32 may be off by: every reference returns (value, size), to be used with layer_ref.within, which allows
160 * 2^-24 * size before the result is rounded.

Activations.  Relative errors: the normal distribution's tail 1.3e-6 by its polynomial and a few 2^-24, the exponential
z^2 * 2^-23 by its argument's two roundings and by that of z; 160 * 2^-24 = 9.5e-6 times 1 + z^2 / 16 covers them.  The logistic
forms: their argument is off by 2^-22 of itself (three roundings, two rounded constants, z), which multiplies the tail:
1 + |argument| / 8.  1 - s is off by 2^-24 whatever it is, so a sixteenth of its factor is added.  Exponentials below 2^-126 may be 0.

Products.  Of 16-bit elements they are exact, of 32-bit ones rounded; a sum of k of them takes k additions in an order that is the
matrix unit's, each off by at most 2^-23 of what its terms add up to in magnitude (it may cut instead of round): k * 2^-23, or
k / 80 times 160 * 2^-24.  Sums of small integers are exact and have to be equal.
"""
import numpy as np
from scipy.special import ndtr

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
FAINT = 2.0 ** -100
C = np.sqrt(2 / np.pi)


def _tanh(z):
    u = 2 * C * (z + 0.044715 * z ** 3)
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-u)), np.abs(u)


def _silu(z):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-z)), np.abs(z)


def act(z, name):
    z = np.asarray(z, np.float64)
    if name == "none":
        return z, np.abs(z)
    if name == "relu":
        return np.where(z <= 0, 0.0, z), np.abs(z)
    if name == "gelu":
        y = z * ndtr(z)
        return y, np.abs(y) * (1 + z * z / 16) + FAINT
    s, u = (_tanh if name == "gelu_tanh" else _silu)(z)
    return z * s, np.abs(z * s) * (1 + u / 8) + FAINT


def slope(z, name):
    z = np.asarray(z, np.float64)
    one = np.ones_like(z)
    if name == "none":
        return one, one
    if name == "relu":
        return np.where(np.isnan(z), z, (z > 0).astype(np.float64)), one
    if name == "gelu":
        p, d = ndtr(z), np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
        return p + z * d, (p + np.abs(z) * d) * (1 + z * z / 16) + FAINT
    if name == "gelu_tanh":
        s, u = _tanh(z)
        g = 2 * C * (1 + 3 * 0.044715 * z * z)
    else:
        s, u = _silu(z)
        g = one
    far = 1 + u / 8
    return s + z * s * (1 - s) * g, s * far + np.abs(z) * s * g * ((1 - s) * far + (u < 40) / 16) + FAINT


def scaled(size, k):
    """The size of a sum of k products whose magnitudes add up to `size`."""
    return size * max(1.0, (k + 64) / 80)


def checkpoint(z):
    """codes, scales of a float32 matrix, in float32 arithmetic: what has to come out bit for bit."""
    z = np.asarray(z, np.float32)
    rows, cols = z.shape
    n = -(-cols // 64)
    wide = np.zeros((rows, n * 64), np.float32)
    wide[:, :cols] = z
    wide = wide.reshape(rows, n, 64)
    with np.errstate(all="ignore"):
        top = np.maximum(np.abs(wide).max(2), np.float32(FAINT))
        bad = ~np.isfinite(wide).all(2)
        scales = np.where(bad, np.float32(np.nan), top / np.float32(127))
        codes = np.rint(wide * (np.float32(127) / top)[:, :, None])
        codes = np.where(bad[:, :, None], 0, codes)
    return codes.reshape(rows, n * 64)[:, :cols].astype(np.int8), scales.astype(np.float32)


def restored(codes, scales):
    """float32: what a checkpoint stands for."""
    return codes.astype(np.float32) * np.repeat(scales, 64, axis=1)[:, :codes.shape[1]]
