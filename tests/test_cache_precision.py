"""The bars of tests/cache_precision.py on a model of the attention (no GPU
needed): probabilities held in fp32, and in 16 bits for bf16 outputs, pass them;
fewer bits do not."""
import functools

import numpy as np
import pytest

import cache_precision as cp
from oracle import cache as oracle


@functools.lru_cache(None)
def reference(dtype, dim, L, sees):
    q, k, v, mask = cp.case(dtype, dim, L, sees)
    assert np.array_equal(oracle.quantise(k), k) and np.array_equal(oracle.quantise(v), v)
    return (q, k, v, mask) + oracle.attend(q, k, v, [L] * len(q), mask, 1.0)[:2]


def model(q, k, v, mask, bits):
    """The attention in 64 bits with probabilities rounded to so many bits, and
    exponents to fp32."""
    out = np.zeros(q.shape)
    for i in range(len(q)):
        ks, vs = k[mask[i]].astype(np.float64), v[mask[i]].astype(np.float64)
        for h in range(q.shape[1]):
            s = (ks[:, h] @ q[i, h].astype(np.float64)) * 1.4426950408889634
            p = 2.0 ** (s - s.max() + 7.0).astype(np.float32).astype(np.float64)
            step = 2.0 ** (np.floor(np.log2(p)) + 1 - bits)
            p = np.round(p / step) * step
            out[i, h] = p @ vs[:, h] / p.sum()
    return out


@pytest.mark.parametrize("dim,L,sees", cp.CASES)
@pytest.mark.parametrize("dtype,bits,passes", [("fp32", 24, True), ("fp32", 22, True), ("fp32", 16, False), ("fp32", 11, False),
                                               ("bf16", 24, True), ("bf16", 16, True), ("bf16", 8, False)])
def test_bars_tell_the_bits(dtype, bits, passes, dim, L, sees):
    q, k, v, mask, ref, mag = reference(dtype, dim, L, sees)
    out = model(q, k, v, mask, bits)
    out = cp.nearest_bf16(out) if dtype == "bf16" else out.astype(np.float32)
    got, bar = cp.misses(dtype, out, ref, mag)
    assert (got <= bar) == passes, (got, bar)
