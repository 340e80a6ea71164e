"""Windows over rows whose counts lie apart: what lies between their windows is
not read, and its table entries may be anything.  Bars as in test_cache_gpu.py."""
import numpy as np
import pytest

from paper_2607_19082_amd import wf
from test_cache_gpu import check, draw, filled, ints
from test_cache_runs_gpu import held, windows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wf.lib()  # fails loudly when the library is missing
    torch.cuda.set_device(0)


def pages_seen(see, page, pages):
    """Of see [B][n][L], [B][pages]: whether any row sees a token of the page."""
    tokens = see.any(1)
    tokens = np.pad(tokens, ((0, 0), (0, pages * page - tokens.shape[1])))
    return tokens.reshape(len(see), pages, page).any(-1)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("counts,L,window,sinks", [
    ([100, 8000], 8000, 64, 0), ([8000, 100, 0, 4000], 8000, 64, 5), ([40, 8000], 8000, 64, 33), ([1, 0, 8000], 8001, 1, 0),
    ([96, 97, 4128, 4129], 4200, 32, 0), ([5, 300, 7000], 7000, 250, 40), ([2000, 2100, 2200], 2200, 100, 0)])
def test_pages_between_windows(counts, L, window, sinks, dtype):
    """Released pages and others' between the windows of one tile's rows; one that
    a single row sees is reported, and left out."""
    dim, page, n = 64, 32, len(counts)
    k, v = draw((1, L, 2, dim), dtype, 1), draw((1, L, 2, dim), dtype, 2)
    see = windows([counts], L, window, sinks)
    hidden = ~see.any((0, 1))
    k[:, hidden], v[:, hidden] = float("nan"), float("inf")
    q = draw((1, n, 4, dim), dtype, 3, 0.0)
    c, table = filled(k, v, page)
    free = torch.from_numpy(~pages_seen(see, page, table.shape[1])).cuda()
    assert free.any()
    table[free] = torch.where(torch.arange(int(free.sum()), device="cuda") % 2 == 0, -1, 1 << 30).int()
    vis = ints([counts])
    out = c.attend_window(q.cuda(), table, vis, window, sinks, max_visible=L)
    c.sync()                                        # nothing is reported
    check(out, q, *held(k, v), [counts], dtype, see)
    assert torch.isfinite(out).all()
    one = (min(m for m in counts if m) - 1) // page
    table[0, one] = -1
    out = c.attend_window(q.cuda(), table, vis, window, sinks, max_visible=L)
    with pytest.raises(wf.WfError) as e:
        c.sync()
    assert e.value.code == wf.WF_E_INVALID
    see[..., one * page:(one + 1) * page] = False
    check(out, q, *held(k, v), [counts], dtype, see)
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,n,hq,heads,dim,L,page,window,sinks", [
    (2, 9, 4, 2, 128, 5000, 32, 20, 4), (1, 16, 1, 1, 64, 20011, 64, 300, 33), (3, 40, 4, 4, 256, 1500, 32, 1, 0), (1, 300, 32, 8, 128, 3000, 32, 9, 40),
    (19, 130, 6, 3, 96, 1000, 32, 5, 0), (4, 520, 8, 8, 64, 2500, 32, 33, 1), (2, 3, 8, 8, 128, 9000, 128, 2000, 300)])
def test_counts_in_no_order(B, n, hq, heads, dim, L, page, window, sinks, dtype):
    """Tiles of 16 and of 32 rows, by workgroups, two waves and one, split and not:
    without the pages that no row sees, a call gives the bits that it gives with
    them, and reports nothing."""
    g = np.random.default_rng(5)
    k, v = draw((B, L, heads, dim), dtype, 1), draw((B, L, heads, dim), dtype, 2)
    q = draw((B, n, hq, dim), dtype, 3, 0.0)
    c, table = filled(k, v, page)
    few = sorted({0, 1, n // 2, n - 1} | set(range(0, n, 1 + n // 7)))
    seqs = sorted({0, B // 2, B - 1})
    near = np.maximum(0, np.array([0, L // 5, L // 2, L])[g.integers(0, 4, (B, n))] - g.integers(0, 3, (B, n)))
    for vis in (near, g.integers(0, L + 1, (B, n))):
        vis[-1, -1], vis[0, 0] = 0, L
        see = np.stack([pages_seen(windows(vis[b:b + 1], L, window, sinks), page, table.shape[1])[0] for b in range(B)])
        want = c.attend_window(q.cuda(), table, ints(vis), window, sinks, max_visible=L)
        c.sync()
        check(want[seqs][:, few], q[seqs][:, few], *held(k[seqs], v[seqs]), vis[seqs][:, few], dtype, windows(vis[seqs][:, few], L, window, sinks))
        released = torch.where(torch.from_numpy(see).cuda(), table, -1)
        assert (released < 0).any() or vis is not near
        out = c.attend_window(q.cuda(), released, ints(vis), window, sinks, max_visible=L)
        c.sync()
        assert torch.equal(out, want)
    c.close()
