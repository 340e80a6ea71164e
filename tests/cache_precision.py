"""Inputs and bars that show how many bits the 4-bit cache's attention keeps of a
probability: scores are sums of two products of modest size, so that they hide
nothing, and a row sees few tokens, so that their errors do not average out.

u = 2^-24.  With |s| <= 2 (times log2 e, less a maximum: at most 13 with the
kernel's lift of 7) the rounded exponent gives a probability of fp32 about 4 u
(rms), exp2, the sums, the joins and the division some 4 more in all: BAR_RMS is
8 u for the root mean square of |out - ref| / A, A = sum p |v| / sum p.
Probabilities of b bits are off by 2^-b at most, sqrt(1/3) of it in the mean of
squares where mantissas are spread: 74 u for 16 bits, of which the three tokens
of a row keep about half, 2400 u for 11.

bf16 outputs are compared with the nearest bf16 of the reference.  Values are not
negative there (A = out), and a relative error e moves an output across a
rounding boundary in a share of about e / 2^-8 of all cases: 16 bits give
40 u / 2^-8 = 0.0006, 8 bits 0.15.  BAR_SHARE lies between.
"""
import numpy as np

U = 2.0 ** -24
BAR_RMS, BAR_SHARE = 8 * U, 0.004
#: dim, tokens, tokens that a row sees
CASES = [(64, 3, 3), (128, 40, 3), (256, 300, 2), (64, 5000, 3), (128, 9001, 3)]


def case(dtype, dim, L, sees, n=16, heads=4):
    """(q, k, v) as float32 arrays [n][heads][dim] and [L][heads][dim] that the
    cache holds exactly (q rounded to bf16 for bf16), and mask [n][L]."""
    g = np.random.default_rng(dim + L + sees)
    q, k = np.zeros((n, heads, dim), np.float32), np.zeros((L, heads, dim), np.float32)
    q[..., [0, dim - 1]] = g.uniform(-1, 1, (n, heads, 2))
    if dtype == "bf16":
        q = (q.view(np.uint32) & 0xffff0000).view(np.float32)
    k[..., [0, dim - 1]] = g.choice([-1.0, -0.5, 0.5, 1.0], (L, heads, 2))
    v = g.choice([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], (L, heads, dim))
    v = v if dtype == "bf16" else v * g.choice([-1, 1], v.shape)
    mask = np.zeros((n, L), bool)
    for i in range(n):
        mask[i, g.choice(L, sees, replace=False)] = True
    return q, k, v.astype(np.float32), mask


def misses(dtype, out, ref, mag):
    """(measure, bar) of outputs against the 64-bit ones and their weighted
    magnitudes."""
    if dtype == "bf16":
        return float((np.asarray(out, np.float64) != nearest_bf16(ref)).mean()), BAR_SHARE
    return float(np.sqrt((((out - ref) / mag) ** 2).mean())), BAR_RMS


def nearest_bf16(x):
    f = np.asarray(x, np.float64)
    step = 2.0 ** (np.floor(np.log2(np.where(f == 0, 1.0, np.abs(f)))) - 7)
    return np.round(f / step) * step
