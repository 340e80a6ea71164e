"""The 4-bit cache's host code on stand-ins for the HIP calls (no GPU needed):
which device and stream its calls use, and what sync reports.  Each test runs in
a process of its own, where the stand-ins (hip_stub.cpp) are loaded before the
library."""
import os
import subprocess
import sys

import pytest

from paper_2607_19082_amd import wf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

START = r'''
import ctypes, sys
sys.path.insert(0, ROOT)
stub = ctypes.CDLL(STUB, mode=ctypes.RTLD_GLOBAL)
from paper_2607_19082_amd import wf
L = wf.lib()
MALLOC, FREE, MEMSET, MEMCPY, MEMCPY_ASYNC, SYNC, LAUNCH, DEVICE_SYNC = range(1, 9)
class Call(ctypes.Structure):
    _fields_ = [("what", ctypes.c_int), ("device", ctypes.c_int), ("stream", ctypes.c_void_p), ("bytes", ctypes.c_uint64),
                ("grid", ctypes.c_uint32), ("block", ctypes.c_uint32)]
num = lambda name: ctypes.c_int.in_dll(stub, name)
def calls(f=None, *args):
    """What a call does: (its return value, the HIP calls)."""
    num("stub_n").value = 0
    rc = f(*args) if f else None
    return rc, list((Call * 4096).in_dll(stub, "stub_calls")[:num("stub_n").value])
def plan(*desc):
    h = ctypes.c_void_p()
    rc, made = calls(L.wf_cache_plan, ctypes.byref(wf.CacheDesc(*desc)), ctypes.byref(h))
    assert rc == 0, L.wf_last_error()
    return h, sum(c.bytes for c in made if c.what == MALLOC)
rows = wf.Rows(0x1000, 1 << 20, 1 << 12, 1 << 8)
P = 0x2000                                          # a device address, never followed
def write(h, B, n, stream=None, pages=64):
    return calls(L.wf_cache_write, h, 1, rows, rows, B, n, P, pages, P, None, stream)
def read(h, B, n, stream=None, pages=64):
    return calls(L.wf_cache_read, h, 1, rows, rows, B, n, P, pages, P, None, stream)
def attend(h, B, n, hq, most, stream=None, precision=1, pages=1 << 15):
    return calls(L.wf_cache_attend, h, precision, rows, rows, B, n, hq, P, pages, P, None, None, most, 1.0, stream)
'''


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    if not os.path.exists(wf.LIB_PATH):
        from paper_2607_19082_amd import build
        build.build()
    d = tmp_path_factory.mktemp("stub")
    stub = str(d / "libstub.so")
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", os.path.join(ROOT, "tests", "hip_stub.cpp"), "-o", stub], check=True)

    def go(code):
        head = f"ROOT, STUB = {ROOT!r}, {stub!r}\n"
        r = subprocess.run([sys.executable, "-c", head + START + code + "\nprint('done')"], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0 and r.stdout.endswith("done\n"), r.stdout + r.stderr

    return go


def test_calls_run_on_the_caches_device(run):
    """A cache of device 1 used while device 0 is current: its launches, and
    what sync does, find device 1 current, and device 0 is current again after."""
    run(r'''
num("stub_device").value = 1
h, _ = plan(8, 128, 64, 64)
num("stub_device").value = 0
for f, args in ((write, (h, 2, 3)), (read, (h, 2, 3)), (attend, (h, 1, 1, 32, 1000)), (attend, (h, 1, 1, 32, 100000))):
    for stream in (None, 0x77):
        rc, made = f(*args, stream=stream)
        assert rc == 0 and made and all(c.what == LAUNCH and c.device == 1 and c.stream == stream for c in made), f
        assert num("stub_device").value == 0
rc, made = calls(L.wf_cache_sync, h, 0x77)
assert rc == 0 and made and all(c.device == 1 for c in made)
assert num("stub_device").value == 0
''')


def test_sync_loses_no_error(run):
    """An error that a kernel on another stream records as soon as sync has
    copied the word is reported by the next sync; all of it goes by the stream
    that sync is given."""
    run(r'''
h, _ = plan(2, 64, 4, 64)
sync = lambda: calls(L.wf_cache_sync, h, 0x77)
num("stub_word").value, num("stub_late").value = 1, 2
rc, made = sync()
assert rc == wf.WF_E_CAPACITY and sync()[0] == wf.WF_E_INVALID and sync()[0] == 0
num("stub_word").value, num("stub_late").value = 0, 1
assert sync()[0] == 0 and sync()[0] == wf.WF_E_CAPACITY and sync()[0] == 0
assert made and all(c.stream == 0x77 for c in made) and made[-1].what == SYNC
''')


def test_token_counts_stay_in_32_bits(run):
    """Calls whose last tiles would end past 2^31 tokens are refused before
    anything is launched; the longest that fits is not."""
    run(r'''
h, _ = plan(1, 64, 4, 1024)
for most in (2**31 - 1, 2**31 - 32, 2**31 - 64):
    rc, made = attend(h, 1, 1, 1, most, pages=1 << 21)
    assert rc == wf.WF_E_UNSUPPORTED and not made, most
assert attend(h, 1, 1, 1, 2**31 - 65, pages=1 << 21)[0] == 0
assert attend(h, 1, 1, 1, 2**31 - 1, pages=1 << 20)[0] == wf.WF_E_INVALID      # more than the table holds
''')


def test_workspace_is_what_calls_take(run):
    """Partial results of split calls, over the workgroups and lengths that the
    split follows from, fit the workspace, and one of them fills it."""
    run(r'''
for dim in (64, 128, 256):
    h, held = plan(1, dim, 64, 64)
    room = held - 256 - 64 * 64 * dim * 17 // 16
    most = 0
    for precision in (0, 1):
        item = 4 - 2 * precision
        for n in list(range(1, 34)) + list(range(48, 340 * 32, 16)):
            for length in (100, 300, 1000, 2100, 8191, 8192, 30000, 131072, 1 << 21):
                rc, made = attend(h, 1, n, 1, length, precision=precision)
                assert rc == 0 and len(made) in (1, 2)
                if len(made) == 2:
                    two = made[0].block == 256 and dim * item < 1024
                    most = max(most, made[0].grid * 16 * (2 if two else 1) * (dim + 2) * 4)
    assert most == room, (dim, most, room)
''')


def test_the_bindings_sync_waits_for_the_caches_device():
    """Cache.sync without a stream waits for the current stream of the cache's
    device, as the calls use it."""
    class Lib:
        def wf_cache_sync(self, handle, stream):
            self.got = getattr(stream, "value", stream)
            return 0

    class Stream:
        cuda_stream = 55

    c = wf.Cache.__new__(wf.Cache)
    c._h, c._device, c._lib, c._current = None, 3, Lib(), lambda device: 1000 + device
    c.sync()
    assert c._lib.got == 1003
    c.sync(Stream)
    assert c._lib.got == 55
