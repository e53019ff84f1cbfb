"""The 8-bit forms in plain numpy, 64 bits, from the definition in include/crisp.h."""
import math

import numpy as np


def exponent(largest):
    """The smallest E >= -126 with largest <= 448 * 2^E."""
    if largest == 0:
        return -126
    e = math.frexp(largest)[1] - 9
    return max(-126, e + (largest > 448.0 * 2.0**e))


def nearest(y):
    """y to the nearest e4m3, even at ties (|y| <= 448); what is not finite becomes NaN."""
    ok = np.isfinite(y)
    z = np.where(ok, y, 0.0)
    _, e = np.frexp(z)
    step = 2.0**(np.maximum(e - 1, -6) - 3)
    return np.where(ok, np.round(z / step) * step, np.nan)


def _largest(a, axis):
    return np.where(np.isfinite(a), np.abs(a), 0.0).max(axis)


def weights(w, mask):
    """float64 [rows, k] and booleans -> what they are held as"""
    rows, k = w.shape
    pad = np.zeros((-(-rows // 128) * 128, -(-k // 128) * 128))
    pad[:rows, :k] = np.where(mask, w, 0.0)
    blocks = pad.reshape(pad.shape[0] // 128, 128, pad.shape[1] // 128, 128)
    scale = 2.0**np.vectorize(exponent)(_largest(blocks, (1, 3))).astype(np.float64)[:, None, :, None]
    return (nearest(blocks / scale) * scale).reshape(pad.shape)[:rows, :k]


def activations(x):
    """float64 [k, ncols] -> what it is held as"""
    k, ncols = x.shape
    pad = np.zeros((-(-k // 128) * 128, ncols))
    pad[:k] = x
    blocks = pad.reshape(-1, 128, ncols)
    scale = 2.0**np.vectorize(exponent)(_largest(blocks, 1)).astype(np.float64)[:, None, :]
    return (nearest(blocks / scale) * scale).reshape(pad.shape)[:k]
