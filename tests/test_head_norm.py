"""The head norm's oracle, its refusals, and its launches on stand-ins for the
HIP calls (no GPU needed)."""
import ctypes

import numpy as np
import pytest

from oracle import head_norm as oracle
from paper_2607_19082_amd import wf
from test_cache_host import run  # noqa: F401 (a fixture)


def test_oracle_norm_and_angles():
    g = np.random.default_rng(0)
    x = g.standard_normal((3, 2, 16))
    y, _ = oracle.head_norm(x, None, eps=0.25)
    assert np.allclose((y ** 2).mean(-1), (x ** 2).mean(-1) / ((x ** 2).mean(-1) + 0.25))
    # near positions agree with 64-bit products, and a turn is a turn
    f = 10000.0 ** (-np.arange(8) / 8)
    p = np.array([0, 1, 17, -5])
    a = oracle.angles(p, f)
    assert np.allclose(np.cos(a), np.cos(p[:, None] * f)) and np.allclose(np.sin(a), np.sin(p[:, None] * f))
    assert (a >= 0).all() and (a < 6.2831854).all()


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_oracle_rotation(pairs):
    """Rotated pairs keep their length, and products of queries with keys
    depend on the distance of positions alone."""
    g = np.random.default_rng(1)
    q, k = g.standard_normal((2, 1, 1, 32))
    f = 100.0 ** (-np.arange(8) / 8)
    go = lambda x, p: oracle.head_norm(x, np.array([p]), frequencies=f, rotated=32, pairs=pairs)[0]  # noqa: E731
    assert np.isclose((go(q, (3, 9)) ** 2).sum(), 32.0, atol=1e-4)
    near, far = (go(q, (3, 9)) * go(k, (1, 4))).sum(), (go(q, (1003, 59)) * go(k, (1001, 54))).sum()
    assert np.isclose(near, far)
    other = (go(q, (3, 9)) * go(k, (1, 5))).sum()
    assert not np.isclose(near, other)


DESC = dict(dim=64, rotated=64, axes=1, pairs=0, eps=1e-6)


def plan(frequencies=None, **change):
    d = DESC | change
    f = np.ones(128) if frequencies is None else np.asarray(frequencies, np.float64)
    h = ctypes.c_void_p()
    rc = wf.lib().wf_head_norm_plan(ctypes.byref(wf.HeadNormDesc(d["dim"], d["rotated"], d["axes"], d["pairs"], d["eps"],
                                                                f.ctypes.data)), ctypes.byref(h))
    assert rc == 0 or not h.value
    return rc


@pytest.mark.parametrize("change,code", [
    (dict(dim=0), wf.WF_E_UNSUPPORTED), (dict(dim=12, rotated=8), wf.WF_E_UNSUPPORTED), (dict(dim=264), wf.WF_E_UNSUPPORTED),
    (dict(axes=0), wf.WF_E_INVALID), (dict(axes=3), wf.WF_E_INVALID), (dict(pairs=2), wf.WF_E_INVALID),
    (dict(rotated=-8), wf.WF_E_INVALID), (dict(rotated=72), wf.WF_E_INVALID), (dict(rotated=20), wf.WF_E_UNSUPPORTED),
    (dict(rotated=24, axes=2), wf.WF_E_UNSUPPORTED), (dict(eps=0.0), wf.WF_E_INVALID), (dict(eps=-1.0), wf.WF_E_INVALID),
    (dict(eps=float("nan")), wf.WF_E_INVALID), (dict(eps=float("inf")), wf.WF_E_INVALID), (dict(eps=1e-39), wf.WF_E_INVALID),
    (dict(frequencies=[7.0] * 32), wf.WF_E_INVALID), (dict(frequencies=[float("nan")] * 32), wf.WF_E_INVALID)])
def test_plans_that_are_refused(change, code):
    assert plan(**change) == code


def test_plan_without_pointers():
    h = ctypes.c_void_p(5)
    assert wf.lib().wf_head_norm_plan(None, ctypes.byref(h)) == wf.WF_E_INVALID and not h.value
    assert wf.lib().wf_head_norm_plan(None, None) == wf.WF_E_INVALID
    wf.lib().wf_head_norm_destroy(None)


NORM = r'''
import numpy as np
f = np.ones(64)
num("stub_device").value = 1
h = ctypes.c_void_p()
rc, made = calls(L.wf_head_norm_plan, ctypes.byref(wf.HeadNormDesc(128, 128, 1, 0, 1e-6, f.ctypes.data)), ctypes.byref(h))
assert rc == 0 and not made              # a plan holds no memory of the device
num("stub_device").value = 0
def norm(B=2, n=3, hq=8, hk=2, q=rows, qo=rows, k=rows, ko=rows, gain=P, positions=P, counts=None, stream=None, precision=1, h=h):
    return calls(L.wf_head_norm, h, precision, q, qo, hq, gain, k, ko, hk, gain, B, n, positions, counts, stream)
'''


def test_calls_that_are_refused(run):  # noqa: F811
    run(NORM + r'''
odd = wf.Rows(0x1001, 1 << 20, 1 << 12, 1 << 8)
for code, args in ((wf.WF_E_INVALID, dict(h=None)), (wf.WF_E_INVALID, dict(precision=2)), (wf.WF_E_INVALID, dict(B=-1)),
                   (wf.WF_E_INVALID, dict(n=-1)), (wf.WF_E_INVALID, dict(hq=0)), (wf.WF_E_INVALID, dict(hk=-1)),
                   (wf.WF_E_INVALID, dict(q=None)), (wf.WF_E_INVALID, dict(qo=None)), (wf.WF_E_INVALID, dict(k=None)),
                   (wf.WF_E_INVALID, dict(ko=None)), (wf.WF_E_INVALID, dict(q=odd)), (wf.WF_E_INVALID, dict(positions=None)),
                   (wf.WF_E_UNSUPPORTED, dict(hq=65537)), (wf.WF_E_UNSUPPORTED, dict(B=1 << 16, n=1 << 15)),
                   (wf.WF_E_UNSUPPORTED, dict(B=1 << 15, n=1 << 15))):
    rc, made = norm(**args)
    assert rc == code and not made, (args, rc)
for args in (dict(B=0), dict(n=0), dict(B=0, q=None, k=None, positions=None)):
    rc, made = norm(**args)
    assert rc == 0 and not made
''')


def test_launches(run):  # noqa: F811
    """Calls run on the plan's device and the given stream; every head of every
    token has a place in the launch."""
    run(NORM + r'''
for stream in (None, 0x77):
    for args in (dict(), dict(k=None, ko=None, hk=0), dict(gain=None), dict(counts=P), dict(precision=0)):
        rc, made = norm(stream=stream, **args)
        assert rc == 0 and len(made) == 1 and made[0].what == LAUNCH and made[0].device == 1 and made[0].stream == stream
        assert num("stub_device").value == 0
for B, n, hq, hk in ((1, 1, 1, 0), (1, 1, 32, 8), (3, 5, 5, 5), (64, 1, 32, 8), (1, 32400, 5, 5), (2, 8191, 32, 8), (1, 100000, 1, 1), (7, 9, 65536, 1)):
    rc, made = norm(B, n, hq, hk)
    assert rc == 0 and len(made) == 1 and made[0].grid >= 1 and made[0].grid * made[0].block < 1 << 32
''')
