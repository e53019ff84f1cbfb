"""Group norm with an activation, forward and backward, in plain numpy, 64 bits, from the definition in include/crisp.h; and how far fp32 sums may be off.

Tolerances count roundings (u = 2^-24 of fp32).  A mean is a sum of values about one of them: the chain of a thread's additions is some 200 long, its roundings are
independent, 16 u of the spread R = max |x - mean| together, and 4 u |mean| for the pieces that are added to it.  M2 is summed the same way, so that rstd is off by 16 u for the
chain, twice (values and pivots), and a few for the root and the division: 48 u of h.  Each elementary step adds its own u."""
import numpy as np

U = 2.0**-24


def grouped(x, groups):
    """[batch, pixels, channels] -> [batch, pixels, groups, channels of one]"""
    return x.reshape(x.shape[0], x.shape[1], groups, -1)


def statistics(x, groups, eps):
    v = grouped(x, groups)
    mean = v.mean((1, 3))
    var = ((v - mean[:, None, :, None])**2).mean((1, 3))
    return mean, 1 / np.sqrt(var + eps)


def spread(a, channels):
    """[batch, groups] -> [batch, 1, channels]"""
    return np.repeat(a, channels // a.shape[1], 1)[:, None]


def act(p, name):
    if name == "relu":
        return np.maximum(p, 0)
    if name == "relu6":
        return np.clip(p, 0, 6)
    return p / (1 + np.exp(-p)) if name == "silu" else p


def slope(p, name):
    if name == "relu":
        return (p > 0) * 1.0
    if name == "relu6":
        return ((p > 0) & (p < 6)) * 1.0
    s = 1 / (1 + np.exp(-p))
    return s + p * s * (1 - s) if name == "silu" else np.ones_like(p)


def forward(x, groups, gamma, beta, eps, name, wide):
    """-> y, mean, rstd, and the tolerance of y before it is rounded.  wide: fp32 (the sigmoid of 16-bit types has 2^-20)"""
    channels = x.shape[2]
    mean, rstd = statistics(x, groups, eps)
    m, r = spread(mean, channels), spread(rstd, channels)
    far = spread(np.abs(grouped(x, groups) - mean[:, None, :, None]).max((1, 3)), channels)
    h = (x - m) * r
    p = gamma * h + beta
    tol = U * (np.abs(gamma) * r * (16 * far + 4 * np.abs(m)) + 48 * np.abs(gamma * h) + 4 * (np.abs(p) + np.abs(beta)))
    y = act(p, name)
    if name == "silu":
        tol = 1.2 * tol + (8 * U if wide else 2.0**-19) * np.abs(y)
    return y, mean, rstd, tol


def backward(dy, x, mean, rstd, groups, gamma, beta, name, wide):
    """-> dx, dgamma, dbeta and their tolerances (dx's before it is rounded)"""
    channels = x.shape[2]
    m, r = spread(mean, channels), spread(rstd, channels)
    h = (x - m) * r
    p = gamma * h + beta
    e = dy * slope(p, name)
    off_h = U * (3 * np.abs(h) + np.abs(m) * r)
    off_e = np.zeros_like(e)
    if name == "silu":                                        # |slope'| <= 1/2
        off_e = np.abs(dy) * (0.5 * (np.abs(gamma) * off_h + 2 * U * (np.abs(p) + np.abs(beta))) + (16 * U if wide else 2.0**-18))
    each = x.shape[1] * channels // groups
    total = lambda a: spread(grouped(a, groups).sum((1, 3)), channels) / each  # noqa: E731
    g = gamma * e
    m1, m2 = total(g), total(g * h)
    off_g = np.abs(gamma) * off_e + U * np.abs(g)
    off_gh = off_g * np.abs(h) + np.abs(g) * off_h + U * np.abs(g * h)
    off1, off2 = (total(o) + 16 * U * total(np.abs(s)) for o, s in ((off_g, g), (off_gh, g * h)))
    dx = r * (g - m1 - h * m2)
    tol = r * (off_g + off1 + np.abs(h) * off2 + off_h * np.abs(m2) + 6 * U * (np.abs(g) + np.abs(m1) + np.abs(h * m2)))
    dbeta, dgamma = e.sum((0, 1)), (e * h).sum((0, 1))
    tol_b = (off_e + 16 * U * np.abs(e)).sum((0, 1))
    tol_g = (off_e * np.abs(h) + np.abs(e) * off_h + 17 * U * np.abs(e * h)).sum((0, 1))
    return dx, dgamma, dbeta, tol, tol_g, tol_b
