"""Attention over the 4-bit cache by a window with first tokens, and behind a
shared prefix, against the oracle.  Bars as in test_cache_gpu.py: a row's tokens
are held and multiplied in the same way whatever run they come from; L is then
all of them."""
import numpy as np
import pytest

from oracle import cache as oracle
from paper_2607_19082_amd import wf
from test_cache_gpu import DTYPE, check, draw, filled, ints

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wf.lib()  # fails loudly when the library is missing
    torch.cuda.set_device(0)


def held(*x):
    return [oracle.quantise(t.float().numpy()) for t in x]


def windows(vis, L, window, sinks):
    """What rows see, [B][n][L]."""
    j, v = np.arange(L), np.asarray(vis)[..., None]
    return (j < v) & ((j >= v - window) | (j < sinks))


# ---- window ----------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256, 40])
@pytest.mark.parametrize("B,n,heads,group,lens,causal,window,sinks", [
    (1, 1, 2, 4, [133], False, 32, 4), (3, 1, 1, 1, [1, 0, 130], False, 1, 0), (2, 5, 2, 3, [170, 64], True, 33, 1),
    (1, 20, 1, 1, [700], True, 100, 0), (2, 9, 1, 7, [257, 31], True, 64, 32), (1, 3, 2, 17, [296], False, 31, 65),
    (1, 2, 1, 1, [300], False, 299, 0), (1, 2, 1, 1, [300], True, 200, 99), (1, 2, 1, 2, [300], False, 5, 1 << 30)])
def test_window(B, n, heads, group, lens, causal, window, sinks, dim, dtype):
    L = max(lens)
    k, v = draw((B, L, heads, dim), dtype, 1), draw((B, L, heads, dim), dtype, 2)
    q = draw((B, n, heads * group, dim), dtype, 3, 0.0)
    c, table = filled(k, v)
    vis = [[max(0, m - (n - 1 - i if causal else 0)) for i in range(n)] for m in lens]
    out = c.attend_window(q.cuda(), table, ints(vis), window, sinks, max_visible=L)
    c.sync()
    check(out, q, *held(k, v), vis, dtype, windows(vis, L, window, sinks))
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,n,group,L,page,window,sinks", [
    (64, 1, 1, 9000, 64, 2000, 4), (128, 1, 8, 9001, 32, 1111, 33), (128, 3, 4, 4050, 128, 3000, 0), (256, 2, 2, 5001, 1024, 1500, 300),
    (64, 40, 1, 6500, 64, 777, 16), (128, 70, 2, 3100, 64, 1000, 64), (128, 600, 4, 900, 64, 300, 5), (64, 515, 8, 500, 32, 33, 40)])
def test_long_windows(dim, n, group, L, page, window, sinks, dtype):
    """Windows split over workgroups, many rows, rows that see unequal prefixes
    in no order, so that one tile's rows are far apart; some see nothing, some
    all there is."""
    g = np.random.default_rng(9)
    heads = 2 if n < 500 else 8
    k, v = draw((2, L, heads, dim), dtype, 1), draw((2, L, heads, dim), dtype, 2)
    q = draw((2, n, heads * group, dim), dtype, 3, 0.0)
    c, table = filled(k, v, page)
    for vis in (np.minimum(L, np.arange(L - n + 1, L + 1)) - np.array([[0], [7]]), g.integers(0, L + 1, (2, n))):
        vis = vis.copy()
        vis[1, -1] = 0
        if n > 2:
            vis[0, 1] = min(L, window + sinks)
            vis[0, 2] = min(L, window + sinks + 1)
        out = c.attend_window(q.cuda(), table, ints(vis), window, sinks, max_visible=L)
        c.sync()
        few = slice(0, None) if n < 100 else slice(0, n, 37)
        check(out[:, few], q[:, few], *held(k, v), vis[:, few], dtype, windows(vis, L, window, sinks)[:, few])
        assert torch.equal(out, c.attend_window(q.cuda(), table, ints(vis), window, sinks, max_visible=L))
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,n", [(64, 1), (128, 3), (256, 2), (128, 20)])
def test_pages_and_values_outside_the_window(dim, n, dtype):
    """Pages that no row sees may be anything, and so may the tokens beside the
    window and the first tokens in the pages that are read."""
    L, window, sinks, page = 1000, 150, 5, 32
    k, v = draw((1, L, 2, dim), dtype, 1), draw((1, L, 2, dim), dtype, 2)
    low = L - n + 1 - window                        # the first token of the window of the row that sees least
    k[:, sinks:low], v[:, sinks:low] = float("nan"), float("inf")
    q = draw((1, n, 4, dim), dtype, 3, 0.0)
    c, table = filled(k, v, page)
    table[0, 1:low // page] = -1
    table[0, 2] = 1 << 30
    vis = [[L - n + 1 + i for i in range(n)]]
    out = c.attend_window(q.cuda(), table, ints(vis), window, sinks, max_visible=L)
    c.sync()                                        # nothing is reported
    check(out, q, *held(k, v), vis, dtype, windows(vis, L, window, sinks))
    assert torch.isfinite(out).all()
    table[0, low // page] = -1                      # a page that rows see is reported, and left out
    out = c.attend_window(q.cuda(), table, ints(vis), window, sinks, max_visible=L)
    with pytest.raises(wf.WfError) as e:
        c.sync()
    assert e.value.code == wf.WF_E_INVALID
    m = windows(vis, L, window, sinks)
    m[..., low // page * page:(low // page + 1) * page] = False
    check(out, q, *held(k, v), vis, dtype, m)
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,n,hq,heads,dim,L,window,sinks", [
    (19, 130, 6, 3, 96, 140, 5, 0), (3, 333, 7, 1, 128, 400, 40, 3), (1, 2100, 8, 8, 64, 2200, 64, 1), (5, 701, 5, 5, 40, 710, 33, 33),
    (2, 260, 16, 2, 256, 300, 20, 2), (1, 1030, 32, 8, 128, 1100, 300, 16), (9, 500, 3, 3, 64, 520, 100, 0)])
def test_many_rows_with_short_windows(B, n, hq, heads, dim, L, window, sinks, dtype):
    """Rows enough that a wave or two take a tile of them, the last workgroup not
    full; causal, and unequal in no order with some that see nothing."""
    g = np.random.default_rng(12)
    k, v = draw((B, L, heads, dim), dtype, 1), draw((B, L, heads, dim), dtype, 2)
    v[:, L // 2, 0, 3] = float("inf")
    q = draw((B, n, hq, dim), dtype, 3, 0.0)
    c, table = filled(k, v)
    few = sorted({0, 1, n // 2, n - 2, n - 1} | set(range(0, n, 1 + n // 13)))
    seqs = sorted({0, B // 2, B - 1})
    for vis in (np.tile(np.arange(L - n + 1, L + 1), (B, 1)), g.integers(0, L + 1, (B, n))):
        vis = vis.copy()
        vis[-1, -1] = vis[0, n // 2] = 0
        out = torch.full_like(q.cuda(), 9.0)
        c.attend_window(q.cuda(), table, ints(vis), window, sinks, max_visible=L, out=out)
        c.sync()
        check(out[seqs][:, few], q[seqs][:, few], *held(k[seqs], v[seqs]), vis[seqs][:, few], dtype, windows(vis, L, window, sinks)[seqs][:, few])
        again = c.attend_window(q.cuda(), table, ints(vis), window, sinks, max_visible=L)
        assert torch.equal(out.nan_to_num(7.0), again.nan_to_num(7.0)) and not (out == 9).all(-1).any()
    c.close()


def test_a_window_that_holds_all_is_attend():
    k, v = draw((2, 500, 2, 64), "bf16", 1), draw((2, 500, 2, 64), "bf16", 2)
    q = draw((2, 3, 4, 64), "bf16", 3, 0.0).cuda()
    c, table = filled(k, v)
    vis = ints([[500, 400, 3], [0, 7, 64]])
    assert torch.equal(c.attend_window(q, table, vis, 500), c.attend(q, table, vis))
    assert torch.equal(c.attend_window(q, table, vis, 2 ** 31 - 1, 2 ** 31 - 1), c.attend(q, table, vis))
    c.close()


# ---- shared prefix ------------------------------------------------------------------


def behind(pk, pv, k, v, page=64, seed=0):
    """A cache that holds the prefix pk, pv [P][heads][dim] and k, v [B][L][..]:
    (cache, the prefix's table, the sequences')."""
    (P, heads, dim), (B, L) = pk.shape, k.shape[:2]
    first, per = -(-P // page), max(1, -(-L // page))
    perm = np.random.default_rng(seed).permutation(first + B * per + 3)
    c = wf.Cache(heads, dim, len(perm), page=page)
    prefix, table = ints(perm[:first]), ints(perm[first:first + B * per].reshape(B, per))
    if P:
        c.write(pk[None].cuda(), pv[None].cuda(), prefix[None], ints([0]))
    if L:
        c.write(k.cuda(), v.cuda(), table, ints([0] * B))
    c.sync()
    return c, prefix, table


def check_shared(out, q, pk, pv, k, v, pvis, vis, dtype, mask=None):
    """Against the oracle: the prefix's tokens and the sequence's own in a row."""
    B, P, L = len(k), len(pk), k.shape[1]
    pk, pv, k, v = held(pk, pv, k, v)
    kk = np.concatenate([np.broadcast_to(pk[None], (B,) + pk.shape), k], 1)
    vv = np.concatenate([np.broadcast_to(pv[None], (B,) + pv.shape), v], 1)
    see = np.concatenate([np.arange(P) < np.asarray(pvis)[..., None], np.arange(L) < np.asarray(vis)[..., None]], -1)
    if mask is not None:
        see &= mask
    check(out, q, kk, vv, np.full(see.shape[:2], P + L), dtype, see)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256, 40])
@pytest.mark.parametrize("B,n,heads,group,P,L,causal", [
    (1, 1, 2, 4, 133, 17, False), (4, 1, 1, 1, 300, 1, False), (5, 2, 2, 3, 64, 70, True), (3, 9, 1, 7, 257, 31, True),
    (17, 1, 2, 4, 1001, 33, False), (2, 33, 1, 1, 65, 40, True), (6, 1, 1, 2, 31, 500, False), (40, 1, 1, 1, 2100, 3, False)])
def test_shared(B, n, heads, group, P, L, causal, dim, dtype):
    """Each row sees all of the prefix; and then unequal parts of it and of its
    own, some none of either."""
    g = np.random.default_rng(4)
    pk, pv = draw((P, heads, dim), dtype, 1), draw((P, heads, dim), dtype, 2)
    k, v = draw((B, L, heads, dim), dtype, 3), draw((B, L, heads, dim), dtype, 4)
    q = draw((B, n, heads * group, dim), dtype, 5, 0.0)
    c, prefix, table = behind(pk, pv, k, v)
    full = np.full((B, n), P)
    for pvis, vis in ((full, np.array([[max(0, L - (n - 1 - i if causal else 0)) for i in range(n)]] * B)),
                      (g.integers(0, P + 1, (B, n)), g.integers(0, L + 1, (B, n))), (full, np.zeros((B, n), int)),
                      (0 * full, np.full((B, n), L))):
        pvis, vis = pvis.copy(), vis.copy()
        if B * n > 3:
            pvis[-1, -1] = 0
            vis[-2:, -1] = 0
        out = torch.full_like(q.cuda(), 9.0)
        c.attend_shared(q.cuda(), prefix, ints(pvis), table, ints(vis), max_prefix=P, max_visible=L, out=out)
        c.sync()
        check_shared(out, q, pk, pv, k, v, pvis, vis, dtype)
        assert torch.equal(out, c.attend_shared(q.cuda(), prefix, ints(pvis), table, ints(vis), max_prefix=P, max_visible=L))
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,B,n,heads,group,P,L,page", [
    (128, 64, 1, 8, 4, 4097, 70, 64), (64, 16, 45, 5, 1, 3001, 90, 64), (128, 8, 64, 2, 4, 2050, 64, 32), (256, 30, 1, 1, 8, 9001, 5, 1024),
    (64, 100, 3, 2, 1, 700, 1500, 128), (96, 2, 300, 8, 2, 500, 300, 64), (8, 700, 1, 4, 2, 333, 40, 32), (8, 3000, 1, 4, 2, 200, 5, 32), (128, 3, 1, 2, 1, 20011, 9000, 64)])
def test_shared_long(dim, B, n, heads, group, P, L, page, dtype):
    """Prefixes split over workgroups, more rows than one launch's workspace
    holds, own tokens that are longer than the prefix; unequal rows."""
    g = np.random.default_rng(6)
    pk, pv = draw((P, heads, dim), dtype, 1), draw((P, heads, dim), dtype, 2)
    k, v = draw((B, L, heads, dim), dtype, 3), draw((B, L, heads, dim), dtype, 4)
    q = draw((B, n, heads * group, dim), dtype, 5, 0.0)
    c, prefix, table = behind(pk, pv, k, v, page)
    pvis, vis = np.full((B, n), P), g.integers(0, L + 1, (B, n))
    pvis[1::3] = g.integers(0, P + 1, pvis[1::3].shape)
    pvis[1], vis[1] = 0, 0
    out = c.attend_shared(q.cuda(), prefix, ints(pvis), table, ints(vis), max_prefix=P, max_visible=L)
    c.sync()
    b = sorted({0, 1, 2, B // 2, B - 2, B - 1} & set(range(B)))
    i = sorted(set(range(0, n, 1 + n // 4)) | {n - 1})
    check_shared(out[b][:, i], q[b][:, i], pk, pv, k[b], v[b], pvis[b][:, i], vis[b][:, i], dtype)
    assert torch.equal(out, c.attend_shared(q.cuda(), prefix, ints(pvis), table, ints(vis), max_prefix=P, max_visible=L))
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,n,group", [(8, 1, 4), (2, 40, 1)])
def test_values_that_rows_do_not_see(B, n, group, dtype):
    """Blocks that are not finite, in the prefix or in a sequence's own tokens,
    change the rows that see them alone; pages outside the pool are left out."""
    P, L, dim, page = 300, 100, 64, 32
    pk, pv = draw((P, 1, dim), dtype, 1), draw((P, 1, dim), dtype, 2)
    k, v = draw((B, L, 1, dim), dtype, 3), draw((B, L, 1, dim), dtype, 4)
    pv[200, 0, 40] = float("nan")
    pk[290:], pv[290:] = float("nan"), float("nan")
    v[1, 50, 0, 7] = float("inf")
    k[:, 90:], v[:, 90:] = float("nan"), float("inf")
    q = draw((B, n, group, dim), dtype, 5, 0.0)
    c, prefix, table = behind(pk, pv, k, v, page)
    pvis, vis = np.full((B, n), 200), np.full((B, n), 90)
    pvis[0], pvis[1, ::2], vis[1, -1] = 290, 100, 50
    out = c.attend_shared(q.cuda(), prefix, ints(pvis), table, ints(vis), max_prefix=P, max_visible=L)
    c.sync()
    check_shared(out, q, pk, pv, k, v, pvis, vis, dtype)
    nan = out.isnan().any(-1).cpu().numpy().any(-1)
    assert nan[0].all() and not nan[2:].any() and (nan[1] == (vis[1] > 50)).all()
    broken, other = prefix.clone(), table.clone()
    broken[3] = -1
    other[B - 1, 1] = 1 << 30
    out = c.attend_shared(q.cuda(), broken, ints(pvis), other, ints(vis), max_prefix=P, max_visible=L)
    with pytest.raises(wf.WfError) as e:
        c.sync()
    assert e.value.code == wf.WF_E_INVALID
    mask = np.ones((B, n, P + L), bool)
    mask[..., 96:128] = False
    mask[B - 1, :, P + 32:P + 64] = False
    check_shared(out, q, pk, pv, k, v, pvis, vis, dtype, mask)
    c.close()


@pytest.mark.parametrize("B,n", [(6, 1), (2, 30)])
def test_rows_that_see_too_much(B, n):
    """Counts beyond what the call allows are cut, and reported; so where the
    call allows no own tokens, or no prefix."""
    P, L = 200, 40
    pk, k, q = draw((P, 1, 64), "fp32", 1), draw((B, L, 1, 64), "fp32", 2), draw((B, n, 2, 64), "fp32", 3).cuda()
    c, prefix, table = behind(pk, pk, k, k)
    many, none = np.full((B, n), 1000), np.zeros((B, n), int)

    def both(pvis, vis, cut_p, cut, max_prefix, max_visible):
        out = c.attend_shared(q, prefix, ints(pvis), table, ints(vis), max_prefix=max_prefix, max_visible=max_visible)
        with pytest.raises(wf.WfError) as e:
            c.sync()
        assert e.value.code == wf.WF_E_CAPACITY
        want = c.attend_shared(q, prefix, ints(cut_p), table, ints(cut), max_prefix=max_prefix, max_visible=max_visible)
        c.sync()
        assert torch.equal(out, want)

    both(many, none + 5, none + 150, none + 5, 150, 20)
    both(none + 100, many, none + 100, none + 20, 150, 20)
    both(none + 100, none + 1, none + 100, none, 150, 0)
    both(none + 1, none + 9, none, none + 9, 0, 20)
    assert (c.attend_shared(q, prefix, ints(none - 3), table, ints(none - 1)) == 0).all()
    w = c.attend_window(q, table, ints(many), 10, 2, max_visible=30)
    with pytest.raises(wf.WfError):
        c.sync()
    assert torch.equal(w, c.attend_window(q, table, ints(none + 30), 10, 2, max_visible=30))
    c.close()


def test_no_prefix_and_no_tokens():
    pk, k, q = draw((100, 2, 64), "bf16", 1), draw((4, 50, 2, 64), "bf16", 2), draw((4, 1, 4, 64), "bf16", 3).cuda()
    c, prefix, table = behind(pk, pk, k, k)
    vis, none = ints([[50], [3], [0], [1]]), ints([[0]] * 4)
    no_table = torch.empty((0,), dtype=torch.int32, device="cuda")
    assert torch.equal(c.attend_shared(q, no_table, none, table, vis), c.attend(q, table, vis))
    every = ints([[100]] * 4)
    no_tables = torch.empty((4, 0), dtype=torch.int32, device="cuda")
    got = c.attend_shared(q, prefix, every, no_tables, none)
    c.sync()
    check(got, q.cpu(), *[np.broadcast_to(x[None], (4,) + x.shape) for x in held(pk, pk)], [[100]] * 4, "bf16")
    assert (c.attend_shared(q, no_table, none, no_tables, none) == 0).all()
    assert c.attend_shared(q[:, :0], prefix, none[:, :0].contiguous(), table, none[:, :0].contiguous()).shape == (4, 0, 4, 64)
    assert c.attend_window(q[:0], table[:0], none[:0], 5).shape == (0, 1, 4, 64)
    c.sync()
    c.close()


# ---- calls ------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_views_streams_and_graphs(dtype):
    """Queries and outputs as views at odd addresses, calls on a stream of their
    own, and a captured step replayed between other work."""
    B, n, P, L, dim = 5, 2, 300, 200, 128
    pk, pv = draw((P, 2, dim), dtype, 1), draw((P, 2, dim), dtype, 2)
    k, v = draw((B, L, 2, dim), dtype, 3), draw((B, L, 2, dim), dtype, 4)
    c, prefix, table = behind(pk, pv, k, v)
    q = draw((B, n, 4, dim), dtype, 5, 0.0)
    wide = torch.full((B, 4, n, 2 * dim + 1), 5.0, dtype=DTYPE[dtype], device="cuda")
    qv, ov = wide[..., 1:dim + 1].transpose(1, 2), wide[..., dim + 1:].transpose(1, 2)
    qv.copy_(q.cuda())
    pvis, vis = ints([[P, P - 1], [0, 7], [P, P], [P, 1], [33, P]]), ints([[150, 151], [3, 0], [0, 0], [L, L - 1], [64, 65]])
    calls = (lambda x, **kw: c.attend_shared(x, prefix, pvis, table, vis, max_prefix=P, max_visible=L, **kw),
             lambda x, **kw: c.attend_window(x, table, vis, 40, 3, max_visible=L, **kw))
    s = torch.cuda.Stream()
    for call in calls:
        want = call(q.cuda())
        s.wait_stream(torch.cuda.current_stream())
        call(qv, out=ov, stream=s)
        c.sync(s)
        assert torch.equal(ov, want) and (wide[..., 0] == 5).all() and torch.equal(qv, q.cuda())
        qs, out, g = q.cuda(), torch.empty_like(want), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            call(qs, out=out)
        for t in range(4):
            qs.mul_(0.7)
            vis.copy_(vis.roll(1, 0))
            out.zero_()
            g.replay()
            got = out.clone()
            torch.cuda.synchronize()
            assert torch.equal(got, call(qs)), t
    c.close()


def test_refusals():
    c = wf.Cache(2, 64, 8, page=32)
    q = torch.zeros((1, 3, 4, 64), device="cuda")
    table, vis, prefix = ints([[0, 1]]), ints([[1, 2, 3]]), ints([2, 3])
    window = lambda **kw: c.attend_window(**(dict(q=q, table=table, visible=vis, window=4) | kw))  # noqa: E731
    shared = lambda **kw: c.attend_shared(**(dict(q=q, prefix_table=prefix, prefix_visible=vis, table=table, visible=vis) | kw))  # noqa: E731
    for kw in (dict(window=0), dict(window=-1), dict(sinks=-1), dict(max_visible=65), dict(scale=0.0)):
        with pytest.raises(wf.WfError) as e:
            window(**kw)
        assert e.value.code == wf.WF_E_INVALID
    for kw in (dict(max_prefix=65), dict(max_prefix=-1), dict(max_visible=65), dict(scale=float("nan"))):
        with pytest.raises(wf.WfError) as e:
            shared(**kw)
        assert e.value.code == wf.WF_E_INVALID
    for kw in (dict(q=q.half()), dict(q=q[0]), dict(table=table.long()), dict(visible=vis[:, :2]), dict(visible=vis.cpu()), dict(out=q[:, :2]),
               dict(window=1 << 31), dict(sinks=1 << 31)):
        with pytest.raises(ValueError):
            window(**kw)
    for kw in (dict(prefix_table=prefix[None]), dict(prefix_table=prefix.long()), dict(prefix_visible=vis[:, :2]), dict(prefix_visible=vis.float()),
               dict(max_prefix=1 << 31), dict(q=q.bfloat16()[..., :32]), dict(table=table[0])):
        with pytest.raises(ValueError):
            shared(**kw)
    c.sync()
    c.close()
