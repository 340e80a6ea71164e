"""Plain 64-bit model of the 4-bit key/value cache and the attention over it.

Written from the format and the formulas alone: a block of 32 consecutive
channels holds values {0, 1/2, 1, 3/2, 2, 3, 4, 6} with a sign times the least
power of two, 2^-125 to 2^125, that makes 6 of it cover the block.
"""
import numpy as np

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def power(top):
    """The least e in [-125, 125] with 6 * 2^e >= top, by search."""
    e = max(-125, min(125, int(np.floor(np.log2(top))) - 6)) if top > 0 else -125
    while e < 125 and 6.0 * 2.0 ** e < top:
        e += 1
    return e


def nearest(y):
    """Index of the grid value nearest to |y|, a tie to the even index."""
    d = np.abs(np.abs(np.asarray(y, np.float64))[..., None] - GRID)
    best = d.min(-1, keepdims=True)
    tied = d == best
    first = tied.argmax(-1)
    two = tied.sum(-1) == 2
    return np.where(two & (first % 2 == 1), first + 1, first)


def quantise(x):
    """The values that the cache holds for x [..., dim]."""
    x = np.asarray(x, np.float64)
    out = np.empty_like(x)
    rows, dst = x.reshape(-1, x.shape[-1]), out.reshape(-1, x.shape[-1])
    for d in range(0, x.shape[-1], BLOCK):
        b = rows[:, d:d + BLOCK]
        top = np.abs(b).max(-1)
        sizes, which = np.unique(np.where(np.isfinite(top), top, 0.0), return_inverse=True)
        p = np.array([2.0 ** power(t) for t in sizes])[which.reshape(-1)][:, None]
        held = GRID[nearest(np.where(np.isfinite(b), b, 0.0) / p)] * np.sign(b) * p
        dst[:, d:d + BLOCK] = np.where(np.isfinite(top)[:, None], held, np.nan)
    return out


def attend(q, k, v, visible, mask=None, scale=None):
    """q [n][hq][D], k and v [L][h][D] (as held), visible [n], mask [n][L]:
    (out, weighted magnitudes sum p |v| / sum p, largest |score| sum) in 64 bits."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, hq, D = q.shape
    G = hq // k.shape[1]
    scale = D ** -0.5 if scale is None else scale
    out, mag, big = np.zeros((n, hq, D)), np.zeros((n, hq, D)), np.zeros((n, hq, 1))
    for i in range(n):
        see = np.arange(len(k)) < visible[i]
        if mask is not None:
            see &= mask[i]
        if not see.any():
            continue
        for h in range(hq):
            ks, vs = k[see, h // G], v[see, h // G]
            s = scale * (ks @ q[i, h])
            p = np.exp(s - s.max())
            out[i, h] = p @ vs / p.sum()
            mag[i, h] = p @ np.abs(vs) / p.sum()
            big[i, h] = scale * (np.abs(ks) @ np.abs(q[i, h])).max()
    return out, mag, big
