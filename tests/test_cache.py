"""The 4-bit cache's host side (no GPU needed): its oracle's own properties and
the descriptions and calls that are refused before any device work."""
import ctypes
import os

import numpy as np
import pytest

from oracle import cache as oracle
from paper_2607_19082_amd import wf


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(wf.LIB_PATH):
        from paper_2607_19082_amd import build
        build.build()
    return wf.lib()


def test_oracle_values():
    """Held values are their own image, errors stay within half a step, and the
    power is the least that covers the block."""
    x = np.random.default_rng(0).standard_normal((200, 70)) * np.exp(np.random.default_rng(1).standard_normal((200, 1)) * 9)
    y = oracle.quantise(x)
    assert np.array_equal(oracle.quantise(y), y)
    for d in range(0, 70, 32):
        b, h = x[:, d:d + 32], y[:, d:d + 32]
        p = 2.0 ** np.array([oracle.power(t) for t in np.abs(b).max(-1)])[:, None]
        assert (np.abs(b) <= 6 * p).all() and (np.abs(b).max(-1, keepdims=True) > 3 * p).all()
        step = np.where(np.abs(b) < 2 * p, 0.5, np.where(np.abs(b) < 4 * p, 1.0, 2.0)) * p
        assert (np.abs(h - b) <= step / 2).all()
    assert np.array_equal(oracle.nearest([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25]), [0, 2, 2, 4, 4, 6, 6, 7, 0])
    assert np.isnan(oracle.quantise([1.0] * 31 + [np.inf])).all()


def test_oracle_attention():
    """Equal scores average, one token passes through, none gives zeros, and a
    mask is the same as leaving the tokens out."""
    g = np.random.default_rng(2)
    k, v, q = g.standard_normal((9, 2, 8)), g.standard_normal((9, 2, 8)), g.standard_normal((4, 6, 8))
    out, _, _ = oracle.attend(q, 0 * k, v, [9, 1, 0, 4])
    assert np.allclose(out[0, 0], v[:, 0].mean(0)) and np.allclose(out[1, 5], v[0, 1]) and (out[2] == 0).all()
    m = g.random((4, 9)) < 0.5
    out, _, _ = oracle.attend(q, k, v, [9] * 4, m)
    for i in range(4):
        one, _, _ = oracle.attend(q[i:i + 1], k[m[i]], v[m[i]], [m[i].sum()])
        assert np.allclose(out[i], one[0])


@pytest.mark.parametrize("desc,code", [
    ((0, 64, 1, 64), wf.WF_E_INVALID), ((1, 64, 0, 64), wf.WF_E_INVALID), ((5000, 64, 1, 64), wf.WF_E_UNSUPPORTED),
    ((1, 0, 1, 64), wf.WF_E_UNSUPPORTED), ((1, 260, 1, 64), wf.WF_E_UNSUPPORTED), ((1, 65, 1, 64), wf.WF_E_UNSUPPORTED),
    ((1, 64, 1, 48), wf.WF_E_UNSUPPORTED), ((1, 64, 1, 16), wf.WF_E_UNSUPPORTED), ((1, 64, 1, 2048), wf.WF_E_UNSUPPORTED)])
def test_descriptions_refused(lib, desc, code):
    h = ctypes.c_void_p(1)
    assert lib.wf_cache_plan(ctypes.byref(wf.CacheDesc(*desc)), ctypes.byref(h)) == code
    assert not h.value and lib.wf_last_error()


def test_null_arguments(lib):
    assert lib.wf_cache_plan(None, ctypes.byref(ctypes.c_void_p())) == wf.WF_E_INVALID
    assert lib.wf_cache_plan(ctypes.byref(wf.CacheDesc(1, 64, 1, 64)), None) == wf.WF_E_INVALID
    r = wf.Rows()
    assert lib.wf_cache_write(None, 0, r, r, 1, 1, None, 1, None, None, None) == wf.WF_E_INVALID
    assert lib.wf_cache_read(None, 0, r, r, 1, 1, None, 1, None, None, None) == wf.WF_E_INVALID
    assert lib.wf_cache_attend(None, 0, r, r, 1, 1, 1, None, 1, None, None, None, 1, 1.0, None) == wf.WF_E_INVALID
    assert lib.wf_cache_sync(None, None) == wf.WF_E_INVALID
    lib.wf_cache_destroy(None)


@pytest.mark.parametrize("desc", [(1, 64, (1 << 32) + 1, 64), ((1 << 32) + 1, 64, 1, 64), (1, 64 - (1 << 32), 1, 64), (1, 64, 1, (1 << 33) + 64)])
def test_sizes_beyond_32_bits_are_refused(lib, desc):
    """ctypes would cut them down to sizes that are fine."""
    with pytest.raises(ValueError):
        wf.Cache(*desc)
