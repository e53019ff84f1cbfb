"""AdamW with states in 32 or 8 bits in plain numpy, 64 bits: what one step makes of given weights, gradients and states, and how a value is
held in the 8-bit forms.  Written from the definition in include/crisp.h."""
import math

import numpy as np

M32 = 0xFFFFFFFF


def mix(h):
    h = np.asarray(h, np.uint64) & M32
    h = h ^ (h >> np.uint64(16))
    h = (h * np.uint64(0x7FEB352D)) & M32
    h = h ^ (h >> np.uint64(15))
    h = (h * np.uint64(0x846CA68B)) & M32
    return h ^ (h >> np.uint64(16))


def hashes(seed, step, tensor, count, first=0):
    """Of `count` elements from number `first` on."""
    key = mix(mix(mix(seed & M32) ^ np.uint64(seed >> 32)) ^ np.uint64(step & M32))
    e = np.arange(first, first + count, dtype=np.uint64)
    return mix((e & np.uint64(M32)) ^ mix((e >> np.uint64(32)) ^ mix(key ^ np.uint64(tensor))))


def decode(codes, biased, root):
    """codes, biased exponents of each 128 -> values (float64)"""
    c = codes.astype(np.int64)
    bits = 4 if root else 3
    field, part = (c >> bits) & 15, c & ((1 << bits) - 1)
    value = np.where(field > 0, (1 + part / 2.0**bits) * 2.0**(field - 7.0), part / 2.0**bits * 2.0**-6)
    if not root:
        value = np.where(c & 128, -value, value)
    return value * 2.0**(np.repeat(biased.astype(np.float64), 128)[:c.size] - 127)


def spacing(y, bits, lowest):
    _, e = np.frexp(np.abs(y))
    return 2.0**(np.maximum(e - 1, lowest) - bits)


def scale_exponents(x, top):
    blocks = np.pad(np.abs(x), (0, -x.size % 128)).reshape(-1, 128).max(1)
    out = np.full(blocks.size, -126)
    for i, a in enumerate(blocks):
        if a > 0:
            e = math.frexp(a)[1] - 9
            out[i] = max(-126, e + (a > top * 2.0**e))
    return out


def hold(x, random, root):
    """(values that are held, the spacing of codes there, exponents)"""
    e = scale_exponents(x, 496.0 if root else 448.0)
    scale = 2.0**np.repeat(e.astype(np.float64), 128)[:x.size]
    y = np.abs(x) / scale
    step = spacing(y, 4 if root else 3, -6)
    code = np.floor(y / step + random)
    if root:
        code = np.where((y > 0) & (code == 0), 1, code)
    return np.sign(x) * code * step * scale, step * scale, e


def step(w, g, m, v, t, mask=None, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, grad_scale=1.0):
    """float64 flat arrays -> new w, m, v, not rounded"""
    g = g * grad_scale
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    w = w * (1 - lr * weight_decay) - lr / (1 - betas[0]**t) * m / (np.sqrt(v) / math.sqrt(1 - betas[1]**t) + eps)
    if mask is not None:
        w, m, v = (np.where(mask, q, 0.0) for q in (w, m, v))
    return w, m, v
