"""Attention behind a shared prefix where the batch is taken in several launches,
and where the rows of all sequences are in tiles of 32 over the prefix: shapes
that test_cache_shapes_host.py holds to that.  Bars as in test_cache_gpu.py."""
import numpy as np
import pytest

from paper_2607_19082_amd import wf
from test_cache_gpu import DTYPE, draw, ints
from test_cache_runs_gpu import behind, check_shared
from test_cache_shapes_host import LAUNCHES, TWO_TILES

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wf.lib()  # fails loudly when the library is missing
    torch.cuda.set_device(0)


def made(dim, B, n, heads, group, P, L, dtype, page=64):
    pk, pv = draw((P, heads, dim), dtype, 1), draw((P, heads, dim), dtype, 2)
    k, v = draw((B, L, heads, dim), dtype, 3), draw((B, L, heads, dim), dtype, 4)
    return pk, pv, k, v, draw((B, n, heads * group, dim), dtype, 5, 0.0), behind(pk, pv, k, v, page)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", LAUNCHES, ids=lambda s: "-".join(map(str, s)))
def test_several_launches(shape, dtype):
    """Queries and outputs are views, so that a launch's first sequence is where its
    strides say; rows on both sides of each launch's end, against the oracle, and
    each sequence against a call of its part alone."""
    dim, B, n, heads, group, P, L, launches = shape
    pk, pv, k, v, q, (c, prefix, table) = made(*shape[:-1], dtype)
    g = np.random.default_rng(8)
    pvis, vis = g.integers(0, P + 1, (B, n)), g.integers(0, L + 1, (B, n))
    pvis[::3] = P
    pvis[5], vis[5] = 0, 0
    hq = heads * group
    wide = torch.full((B, n + 1, 2 * hq, dim + 1), 5.0, dtype=DTYPE[dtype], device="cuda")
    qv, out = wide[:, :n, :hq, 1:], wide[:, 1:, hq:, :dim]
    qv.copy_(q.cuda())
    before = wide.clone()
    c.attend_shared(qv, prefix, ints(pvis), table, ints(vis), max_prefix=P, max_visible=L, out=out)
    c.sync()
    got = out.clone()
    out.fill_(5.0)
    assert torch.equal(wide, before)                    # nothing beside the outputs
    part = -(-B // launches)
    ends = [x for i in range(1, launches) for x in (i * part - 1, i * part)]
    some = sorted({0, 1, 5, B // 3, B - 2, B - 1} | set(ends))
    check_shared(got[some], q[some], pk, pv, k[some], v[some], pvis[some], vis[some], dtype)
    assert (got[5] == 0).all()
    for a in range(0, B, part):                         # the same launches, one by one
        s = slice(a, min(B, a + part))
        one = c.attend_shared(q[s].cuda(), prefix, ints(pvis[s]), table[s], ints(vis[s]), max_prefix=P, max_visible=L)
        few = list(range(0, part, 97)) + [len(one) - 1]
        few = [x for x in few if x < len(one)]
        check_shared(one[few], q[s][few], pk, pv, k[s][few], v[s][few], pvis[s][few], vis[s][few], dtype)
    assert torch.equal(got, c.attend_shared(q.cuda(), prefix, ints(pvis), table, ints(vis), max_prefix=P, max_visible=L))
    c.sync()
    c.close()


@pytest.mark.parametrize("shape,dtype", [(s[:-1], "bf16" if p else "fp32") for s in TWO_TILES for p in s[-1]],
                         ids=lambda s: s if isinstance(s, str) else "-".join(map(str, s)))
def test_tiles_of_32_rows_over_the_prefix(shape, dtype):
    """Rows of several sequences in a tile, a sequence's own that end within a tile;
    all of the prefix, then unequal parts of it and of their own, some none."""
    dim, B, n, heads, group, P, L = shape
    pk, pv, k, v, q, (c, prefix, table) = made(*shape, dtype)
    g = np.random.default_rng(9)
    own = np.maximum(0, L - np.arange(n)[::-1] % 40)[None] if L else np.zeros((1, n), int)
    for pvis, vis in ((np.full((B, n), P), np.repeat(own, B, 0)), (g.integers(0, P + 1, (B, n)), g.integers(0, L + 1, (B, n)))):
        pvis, vis = pvis.copy(), vis.copy()
        pvis[2, n // 2] = vis[2, n // 2] = 0
        pvis[B - 1, -1] = vis[0, 0] = 0
        out = torch.full_like(q.cuda(), 9.0)
        c.attend_shared(q.cuda(), prefix, ints(pvis), table, ints(vis), max_prefix=P, max_visible=L, out=out)
        c.sync()
        b = [0, 1, 2, B // 2, B - 1]
        i = sorted({0, 1, n // 2, n - 2, n - 1})
        check_shared(out[b][:, i], q[b][:, i], pk, pv, k[b], v[b], pvis[b][:, i], vis[b][:, i], dtype)
        assert (out[2, n // 2] == 0).all() and not (out == 9).all(-1).any()
        assert torch.equal(out, c.attend_shared(q.cuda(), prefix, ints(pvis), table, ints(vis), max_prefix=P, max_visible=L))
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_values_that_are_not_finite_in_tiles_of_32_rows(dtype):
    """They change the rows that see them alone."""
    dim, B, n, heads, group, P, L = TWO_TILES[1][:-1]
    pk, pv, k, v, q, (c, prefix, table) = made(dim, B, n, heads, group, P, L, dtype)
    c.close()
    pv[8000, 0, 40] = float("nan")
    pk[8990:], pv[8990:] = float("nan"), float("inf")
    v[3, 20, 0, 7] = float("inf")
    c, prefix, table = behind(pk, pv, k, v)
    pvis, vis = np.full((B, n), 8000), np.full((B, n), 20)
    pvis[1], vis[3, ::2], pvis[4, -1] = 8001, 21, P
    out = c.attend_shared(q.cuda(), prefix, ints(pvis), table, ints(vis), max_prefix=P, max_visible=L)
    c.sync()
    some = [0, 1, 3, 4, B - 1]
    check_shared(out[some], q[some], pk, pv, k[some], v[some], pvis[some], vis[some], dtype)
    nan = out.isnan().any(-1).any(-1).cpu().numpy()
    want = (pvis > 8000) | (vis > 20)
    assert (nan == want).all()
    c.close()
