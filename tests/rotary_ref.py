"""Norm and rotation of rows in 64 bits, and how far single precision may be off it."""
import numpy as np


def turned(x, angle, layout, begin, rot, amplitude=1.0):
    """x float64 [B][H][n][d], angle float64 [B][n][rot / 2] in radians."""
    y = x.copy()
    c, s = amplitude * np.cos(angle)[:, None], amplitude * np.sin(angle)[:, None]
    i = np.arange(rot // 2)
    u, v = (begin + i, begin + i + rot // 2) if layout == 0 else (begin + 2 * i, begin + 2 * i + 1)
    y[..., u] = x[..., u] * c - x[..., v] * s
    y[..., v] = x[..., v] * c + x[..., u] * s
    return y


def normed(x, kind, eps, weight, bias):
    """weight, bias float64, broadcast over [B][H][n][d]."""
    if kind == 0:
        return x.copy()
    if kind == 2:
        x = x - x.mean(-1, keepdims=True)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight + bias


def angles(turns, pos):
    """turns uint64 [half], pos int64 [..., half] -> radians; the fraction of a turn is exact in 64 bits."""
    with np.errstate(over="ignore"):
        fraction = pos.astype(np.int64).view(np.uint64) * turns
    return fraction.view(np.int64).astype(np.float64) * (2.0 * np.pi / 2.0 ** 64)


def bound(x, y, weight, bias, kind, eps, layout, begin, rot, amplitude, out_eps):
    """Largest difference of each output from 64 bits.  x: the inputs, y: after the norm (both float64).

    u = 2^-24.  Norm: a lane adds at most 16 squares, its group 6 times more: the sum is off by 22 u, its mean by two roundings more, the root halves that
    (12 u); root, reciprocal and two products add 5: 17 u of y - bias, the sum with the bias u of y.  With a mean taken out: the mean is off by 23 u of the
    mean magnitude, the difference by u more of the largest (24 u), once in y and once, at most as much, through the variance: 48 u max|x| / deviation.
    Rotation: sine and cosine within 2^-23 (2 u) and the angle's last place (2^-32 turns: 2^-29.3, below u / 16), times amplitude u, a product and a sum u each: 5.1 u of
    |a| + |b|, times the amplitude.  Then the output's own rounding."""
    u = 2.0 ** -24
    e = np.zeros_like(y)
    if kind:
        e = 17 * u * np.abs(y - bias) + u * np.abs(y)
    if kind == 2:
        centred = x - x.mean(-1, keepdims=True)
        e = e + 48 * u * np.abs(x).max(-1, keepdims=True) / np.sqrt((centred ** 2).mean(-1, keepdims=True) + eps) * np.abs(weight)
    e = np.broadcast_to(e, y.shape).copy()
    size = np.abs(y) + e
    i = np.arange(rot // 2)
    a, b = (begin + i, begin + i + rot // 2) if layout == 0 else (begin + 2 * i, begin + 2 * i + 1)
    pair = amplitude * ((e[..., a] + e[..., b]) + 5.1 * u * (size[..., a] + size[..., b]))
    e[..., a] = pair
    e[..., b] = pair
    return e * (1 + out_eps) + 2.0 ** -140, out_eps
