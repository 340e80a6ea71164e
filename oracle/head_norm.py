"""Plain 64-bit model of the head norm with position rotation.

Written from the formulas alone; angles are reduced to one turn in exact
arithmetic before their sines are taken, so that no position is too far.
"""
from fractions import Fraction

import numpy as np

#: pi to 50 places
PI = Fraction(314159265358979323846264338327950288419716939937511, 10 ** 50)


def angles(positions, frequencies):
    """positions (any shape) times frequencies [pairs], radians modulo a turn."""
    positions = np.asarray(positions, np.int64)
    out = np.empty(positions.shape + (len(frequencies),))
    distinct = {}
    for at in np.ndindex(positions.shape):
        p = int(positions[at])
        if p not in distinct:
            turns = [Fraction(float(f)) * p / (2 * PI) for f in frequencies]
            distinct[p] = [float((t - (t.numerator // t.denominator)) * 2 * PI) for t in turns]
        out[at] = distinct[p]
    return out


def head_norm(x, positions, gain=None, eps=1e-6, frequencies=None, rotated=0, pairs="halves"):
    """x [..., heads, dim], positions [..., axes] -> (rows, the magnitude of each
    channel's pair), in 64 bits."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if gain is not None:
        y = y * np.asarray(gain, np.float64)
    size = np.abs(y)
    if not rotated:
        return y, size
    axes = positions.shape[-1]
    part = rotated // axes
    z = y.copy()
    for axis in range(axes):
        t = angles(positions[..., axis], frequencies)[..., None, :]
        at = np.arange(part // 2)
        if pairs == "halves":
            a, b = axis * part + at, axis * part + part // 2 + at
        else:
            a, b = axis * part + 2 * at, axis * part + 2 * at + 1
        z[..., a] = y[..., a] * np.cos(t) - y[..., b] * np.sin(t)
        z[..., b] = y[..., a] * np.sin(t) + y[..., b] * np.cos(t)
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return z, size
