"""Host code of the windowed and the shared attention on stand-ins for the HIP
calls (no GPU needed)."""
from paper_2607_19082_amd import wf  # noqa: F401 (built by the fixture below)
from test_cache_host import run  # noqa: F401 (a fixture)

CALLS = r'''
def window(h, B, n, hq, most, window, sinks, stream=None, precision=1, pages=1 << 15, q=rows, vis=P):
    return calls(L.wf_cache_attend_window, h, precision, q, rows, B, n, hq, P, pages, vis, window, sinks, most, 1.0, stream)
def shared(h, B, n, hq, prefix, most, stream=None, precision=1, first_pages=1 << 15, pages=1 << 15, table=P, vis=P):
    return calls(L.wf_cache_attend_shared, h, precision, rows, rows, B, n, hq, table, first_pages, vis, prefix, P, pages, P, most, 1.0, stream)
'''


def test_refusals(run):  # noqa: F811
    run(CALLS + r'''
h, _ = plan(2, 64, 4, 1024)
for bad in (dict(window=0, sinks=0), dict(window=-5, sinks=0), dict(window=5, sinks=-1), dict(window=5, sinks=0, q=None),
            dict(window=5, sinks=0, vis=None), dict(window=5, sinks=0, precision=3), dict(window=5, sinks=0, pages=0)):
    rc, made = window(h, 1, 1, 2, 100, **bad)
    assert rc == wf.WF_E_INVALID and not made, bad
assert window(None, 1, 1, 2, 100, 5, 0)[0] == wf.WF_E_INVALID
assert window(h, 1, 1, 3, 100, 5, 0)[0] == wf.WF_E_INVALID
assert window(h, 0, 1, 2, 100, 5, 0) == (0, []) and window(h, 1, 0, 2, 100, 5, 0) == (0, [])
for bad in (dict(prefix=-1, most=5), dict(prefix=5, most=-1), dict(prefix=1025, most=5, first_pages=1), dict(prefix=5, most=5, first_pages=-1),
            dict(prefix=5, most=5, table=None), dict(prefix=5, most=5, vis=None), dict(prefix=5, most=1025, pages=1)):
    rc, made = shared(h, 2, 1, 2, **bad)
    assert rc == wf.WF_E_INVALID and not made, bad
assert shared(None, 2, 1, 2, 5, 5)[0] == wf.WF_E_INVALID
assert shared(h, 0, 1, 2, 5, 5) == (0, []) and shared(h, 1, 0, 2, 5, 5) == (0, [])
# token counts stay in 32 bits
big = dict(first_pages=1 << 21, pages=1 << 21)
assert shared(h, 2, 1, 2, 2**31 - 1 - 128 - 100, 100, **big)[0] == 0
for p, m in ((2**31 - 128 - 100, 100), (2**31 - 1, 2**31 - 65), (1, 2**31 - 65), (2**31 - 1, 0)):
    rc, made = shared(h, 2, 1, 2, p, m, **big)
    assert rc == wf.WF_E_UNSUPPORTED and not made, (p, m)
assert window(h, 1, 1, 2, 2**31 - 64, 2**31 - 1, 2**31 - 1, pages=1 << 21)[0] == wf.WF_E_UNSUPPORTED
for w, s in ((2**31 - 1, 2**31 - 1), (1, 2**31 - 1), (2**31 - 1, 0), (5, 5)):
    assert window(h, 1, 1, 2, 2**31 - 65, w, s, pages=1 << 21)[0] == 0
''')


def test_device_and_stream(run):  # noqa: F811
    run(CALLS + r'''
num("stub_device").value = 1
h, _ = plan(8, 128, 64, 64)
num("stub_device").value = 0
for f, args in ((window, (h, 1, 1, 32, 10000, 4000, 4)), (window, (h, 64, 1, 32, 10000, 100, 0)), (shared, (h, 64, 1, 32, 8192, 700)),
                (shared, (h, 8, 128, 32, 8192, 128)), (shared, (h, 2000, 1, 32, 8192, 50)), (shared, (h, 4, 1, 8, 100, 0))):
    for stream in (None, 0x77):
        rc, made = f(*args, stream=stream)
        assert rc == 0 and made and all(c.what == LAUNCH and c.device == 1 and c.stream == stream for c in made), f
        assert num("stub_device").value == 0
''')


def test_partial_results_fit_the_workspace(run):  # noqa: F811
    """Launches that leave partial results (a join follows them) leave no more
    than the workspace holds, whatever the rows, heads and lengths."""
    run(CALLS + r'''
most = 0
for dim in (64, 128, 256):
    for heads in (1, 5, 64, 1000):
        h, held = plan(heads, dim, 4, 32)
        room = held - 256 - (4 * 32 * heads * dim * 17 // 16 + 255) // 256 * 256
        for precision in (0, 1):
            item = 4 - 2 * precision
            for group in (1, 4, 16):
                for B, n in ((1, 1), (2, 1), (3, 7), (8, 128), (64, 1), (16, 45), (333, 2), (5000, 1), (20, 1000), (40000, 1)):
                    if B * n * heads * group > 1 << 22:
                        continue
                    for f, args in [(shared, (x, y)) for x in (31, 1000, 8192, 131072) for y in (0, 1, 777, 20000)] + \
                            [(window, (20000, w, 4)) for w in (50, 5000)]:
                        rc, made = f(h, B, n, heads * group, *args, precision=precision)
                        assert rc == 0 and (len(made) == 1 or len(made) % 2 == 0)
                        if len(made) > 1:               # each launch and its join
                            launches = len(made) // 2
                            part, left = -(-B // launches), B
                            for c in made[::2]:
                                tile = 32 if c.block == 256 and dim * item < 1024 else 16
                                fits = c.grid * tile * (dim + 2) * 4 <= room
                                if f is shared and not fits:
                                    # rows of all over the prefix, in tiles, and each sequence's over its own, in rows
                                    b, r = min(part, left), n * group
                                    first, own = heads * -(-b * r // tile), b * heads * -(-r // tile) if args[1] else 0
                                    fits = any((s * first * tile + (c.grid - s * first) * min(r, tile)) * (dim + 2) * 4 <= room
                                               and (c.grid - s * first) % max(1, own) == 0 for s in range(1, c.grid // first + 1))
                                assert fits, (dim, heads, precision, group, B, n, args)
                                left -= part
                            most = max(most, len(made))
        L.wf_cache_destroy(h)
assert most > 8                                         # batches that are taken in parts
''')
