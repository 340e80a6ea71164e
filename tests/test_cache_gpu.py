"""The 4-bit key/value cache on the GPU: what is written reads back as the
oracle's values exactly, and the attention over it agrees with 64 bits.

Bars of the attention, derived from its arithmetic (u = 2^-24, D channels, L
tokens, S = the largest scale * sum |q k| of a row, A = sum p |v| / sum p):
 - a score is a sum of D exact products of parts in fp32: off by (D + 4) u S at
   most (the scale's and the exponent's own roundings among the four), so a
   probability by twice that, and their sums by (L + 64) u;
 - bf16 calls hold a probability to 2^-16 and round the output to 2^-8.
Worst cases, added: |got - ref| <= A (2 (D + 4) S + 2 (L + 64)) u (+ A 2^-15 +
2^-8 |ref| for bf16).
"""
import numpy as np
import pytest

from oracle import cache as oracle
from paper_2607_19082_amd import wf

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wf.lib()  # fails loudly when the library is missing
    torch.cuda.set_device(0)


DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


def draw(shape, dtype, seed, spread=0.7):
    """Channels of unequal size with an offset, as keys have them."""
    g = np.random.default_rng(seed)
    x = g.standard_normal(shape) * np.exp(spread * g.standard_normal(shape[-1])) + 0.3 * g.standard_normal(shape[-1])
    return torch.from_numpy(x.astype(np.float32)).to(DTYPE[dtype])


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def pages_of(B, tokens, page, seed=0, spare=3):
    """A shuffled page table for B sequences, and the pool's pages."""
    per = max(1, -(-tokens // page))
    perm = np.random.default_rng(seed).permutation(B * per + spare)[:B * per]
    return ints(perm.reshape(B, per)), B * per + spare


def filled(k, v, page=64, seed=0):
    """A cache that holds k and v [B][L][heads][dim] (host tensors) from token 0."""
    B, L, h, D = k.shape
    table, pages = pages_of(B, L, page, seed)
    c = wf.Cache(h, D, pages, page=page)
    c.write(k.cuda(), v.cuda(), table, ints([0] * B))
    c.sync()
    return c, table


# ---- write and read --------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,n,heads,dim,page", [(1, 1, 1, 64, 32), (2, 45, 5, 64, 64), (3, 33, 2, 128, 32),
                                                (1, 130, 3, 256, 64), (2, 7, 2, 96, 128), (1, 70, 4, 40, 64),
                                                (1, 40, 1, 8, 32), (2, 65, 2, 200, 1024)])
def test_round_trip(B, n, heads, dim, page, dtype):
    k, v = draw((B, n, heads, dim), dtype, 1), draw((B, n, heads, dim), dtype, 2)
    c, table = filled(k, v, page)
    for out in ("fp32", dtype):
        gk, gv = c.read(table, ints([0] * B), n, dtype=DTYPE[out])
        c.sync()
        for got, x in ((gk, k), (gv, v)):
            assert np.array_equal(got.float().cpu().numpy(), oracle.quantise(x.float().numpy()).astype(np.float32))
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_values_at_the_edges(dtype):
    """Zeros, ties, the powers' ends, magnitudes beyond the largest power, and
    blocks with values that are not finite, each in a block of its own."""
    g = np.random.default_rng(5)
    blocks = [np.zeros(32), -np.zeros(32)]
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for p in (-125, -60, 0, 9, 125):
        blocks.append(np.concatenate([ties, -ties, ties * (1 + 2.0 ** -7), -ties * (1 - 2.0 ** -7)]).clip(-6, 6) * 2.0 ** p)
    for top in (3.0, 3.0 * (1 + 2.0 ** -7), 6.0, 6.0 * (1 + 2.0 ** -7), 5.98):
        blocks.append(g.uniform(-1, 1, 32) * top)
        blocks[-1][g.integers(32)] = top
    blocks.append(g.standard_normal(32) * 2.0 ** -125)
    blocks.append(g.standard_normal(32) * 2.0 ** -126)
    blocks.append(np.full(32, 3.3e38) * np.sign(g.standard_normal(32)))
    for bad in (np.nan, np.inf, -np.inf):
        blocks.append(g.standard_normal(32))
        blocks[-1][g.integers(32)] = bad
    while len(blocks) % 4:
        blocks.append(g.standard_normal(32))
    x = torch.from_numpy(np.stack(blocks).reshape(1, -1, 1, 128).astype(np.float32)).to(DTYPE[dtype])
    c, table = filled(x, x.flip(1))
    gk, gv = c.read(table, ints([0]), x.shape[1])
    want = oracle.quantise(x.float().numpy()).astype(np.float32)
    assert np.array_equal(gk.cpu().numpy(), want, equal_nan=True)
    assert np.array_equal(gv.cpu().numpy(), want[:, ::-1], equal_nan=True)
    assert np.isnan(want).sum() == 96
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_tokens_are_their_own(dim, dtype):
    """Tokens written one at a time, out of order and across pages, from views
    of a wider array at odd addresses, leave every other token as it was."""
    B, L, heads, page = 2, 75, 2, 32
    wide = draw((B, L, 2 * heads + 1, dim + 3), dtype, 3).cuda()
    k, v = wide[:, :, :heads, 1:dim + 1], wide[:, :, heads + 1:, 2:dim + 2]
    table, pages = pages_of(B, L, page)
    c = wf.Cache(heads, dim, pages, page=page)
    want = np.zeros((2, B, L, heads, dim), np.float32)
    order = np.random.default_rng(0).permutation(L)
    for step, t in enumerate(order):
        at = [int(t), int((t + 40) % L)]
        c.write(torch.stack([k[b, at[b]] for b in range(B)])[:, None], torch.stack([v[b, at[b]] for b in range(B)])[:, None],
                table, ints(at), counts=ints([1, step % 2]))
        for b in range(B):
            if b == 0 or step % 2:
                want[0, b, at[b]] = oracle.quantise(k[b, at[b]].float().cpu().numpy())
                want[1, b, at[b]] = oracle.quantise(v[b, at[b]].float().cpu().numpy())
    gk, gv = c.read(table, ints([0, 0]), L)
    c.sync()
    assert np.array_equal(gk.cpu().numpy(), want[0]) and np.array_equal(gv.cpu().numpy(), want[1])
    # a view as the source of a whole write, and views as the destination of a read
    c.write(k, v, table, ints([0, 0]))
    out = torch.full((B, L, heads, 2, dim + 1), 7.0, dtype=DTYPE[dtype], device="cuda")
    c.read(table, ints([3, 0]), L - 3, counts=ints([L - 3, 5]), out=(out[:, :L - 3, :, 0, 1:], out[:, :L - 3, :, 1, 1:]))
    c.sync()
    for j, x in enumerate((k, v)):
        want = oracle.quantise(x.float().cpu().numpy()).astype(np.float32)
        got = out[:, :, :, j].float().cpu().numpy()
        assert np.array_equal(got[0, :L - 3, :, 1:], want[0, 3:])
        assert np.array_equal(got[1, :5, :, 1:], want[1, :5])
        assert (got[1, 5:L - 3, :, 1:] == 0).all()
        assert (got[..., 0] == 7).all() and (got[:, L - 3:] == 7).all()
    c.close()


def test_pool_beyond_4_gib():
    """Pages whose bytes lie past 2^32 in the pool."""
    heads, dim, page = 8, 256, 1024
    pages = (1 << 32) // (page * heads * dim * 17 // 16) + 8
    c = wf.Cache(heads, dim, pages, page=page)
    k, v = draw((1, 40, heads, dim), "bf16", 1), draw((1, 40, heads, dim), "bf16", 2)
    q = draw((1, 2, heads, dim), "bf16", 3, 0.0)
    table = ints([[pages - 1, 0, pages - 2]])
    c.write(k.cuda(), v.cuda(), table, ints([1000]))
    gk, gv = c.read(table, ints([1000]), 40)
    mask = torch.zeros((1, 2, 1040), dtype=torch.bool, device="cuda")
    mask[:, :, 1000:] = True
    out = c.attend(q.cuda(), table, ints([[1040, 1030]]), mask=mask)
    c.sync()
    kq, vq = oracle.quantise(k.float().numpy()), oracle.quantise(v.float().numpy())
    assert np.array_equal(gk.cpu().numpy(), kq.astype(np.float32)) and np.array_equal(gv.cpu().numpy(), vq.astype(np.float32))
    check(out, q, kq, vq, [[40, 30]], "bf16")
    c.close()


# ---- attention -------------------------------------------------------------------


def check(out, q, kq, vq, visible, dtype, mask=None, scale=None):
    """out against the oracle on the held values kq, vq [B][L][heads][dim]."""
    out, q = out.float().cpu().numpy().astype(np.float64), q.float().cpu().numpy()
    D, L = q.shape[-1], kq.shape[1]
    for b in range(len(q)):
        ref, mag, big = oracle.attend(q[b], kq[b], vq[b], visible[b], None if mask is None else mask[b], scale)
        tol = mag * (2 * (D + 4) * big + 2 * (L + 64)) * U
        if dtype == "bf16":
            tol = tol + mag * 2.0 ** -15 + np.abs(ref) * 2.0 ** -8
        assert np.array_equal(np.isnan(out[b]), np.isnan(ref)), b
        far = np.abs(out[b] - ref) - tol
        assert not (far > 0).any(), (b, float(np.nanmax(far)), np.argwhere(far > 0)[:5])
        assert (out[b][mag.sum(-1) == 0] == 0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256, 40, 96, 200])
@pytest.mark.parametrize("B,n,heads,group,lens,causal", [
    (1, 1, 2, 4, [33], False), (3, 1, 1, 1, [1, 0, 130], False), (2, 5, 2, 3, [70, 64], True),
    (1, 20, 1, 1, [700], True), (2, 9, 1, 7, [257, 31], True), (1, 3, 2, 17, [96], False)])
def test_attend(B, n, heads, group, lens, causal, dim, dtype):
    L = max(lens)
    k, v = draw((B, L, heads, dim), dtype, 1), draw((B, L, heads, dim), dtype, 2)
    q = draw((B, n, heads * group, dim), dtype, 3, 0.0)
    c, table = filled(k, v)
    vis = [[max(0, m - (n - 1 - i if causal else 0)) for i in range(n)] for m in lens]
    out = c.attend(q.cuda(), table, ints(vis))
    c.sync()
    check(out, q, oracle.quantise(k.float().numpy()), oracle.quantise(v.float().numpy()), vis, dtype)
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,n,group,L,page", [(64, 1, 1, 5000, 64), (128, 1, 8, 4097, 32), (128, 3, 4, 2050, 128),
                                                (256, 2, 2, 3001, 1024), (64, 40, 1, 2500, 64), (128, 70, 2, 1100, 64)])
def test_attend_long(dim, n, group, L, page, dtype):
    """Tokens split over workgroups, rows over several tiles; rows see unequal
    prefixes in no order, some nothing."""
    g = np.random.default_rng(9)
    k, v = draw((2, L, 2, dim), dtype, 1), draw((2, L, 2, dim), dtype, 2)
    q = draw((2, n, 2 * group, dim), dtype, 3, 0.0)
    c, table = filled(k, v, page)
    vis = g.integers(0, L + 1, (2, n))
    vis[0, 0] = L
    vis[1, -1] = 0
    out = c.attend(q.cuda(), table, ints(vis), max_visible=L)
    c.sync()
    check(out, q, oracle.quantise(k.float().numpy()), oracle.quantise(v.float().numpy()), vis, dtype)
    again = c.attend(q.cuda(), table, ints(vis), max_visible=L)
    assert torch.equal(out, again)                  # the order of sums follows from the sizes
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,n,heads,group,lens", [
    (64, 1, 3, 1, [5000, 0, 3, 0, 0, 33, 700, 1]), (128, 1, 2, 4, [0, 0, 900, 64, 2100]), (256, 2, 1, 3, [300, 301, 0]),
    (128, 3, 1, 5, [40] * 50 + [1500] + [0] * 20), (64, 2, 2, 1, [0, 0]), (128, 1, 1, 16, [1024] * 6),
    (96, 1, 1, 8, list(range(0, 400, 7))), (64, 1, 8, 1, [17] * 256)])
def test_batches_of_any_lengths(dim, n, heads, group, lens, dtype):
    """A token or two of many sequences: one long among short ones, none, equal
    ones, as many as a launch takes together."""
    B, L = len(lens), max(max(lens), 1)
    g = np.random.default_rng(3)
    k, v = draw((B, L, heads, dim), dtype, 1), draw((B, L, heads, dim), dtype, 2)
    q = draw((B, n, heads * group, dim), dtype, 3, 0.0)
    c, table = filled(k, v)
    vis = np.array([[m if i == 0 else g.integers(0, m + 1) for i in range(n)] for m in lens])
    out = torch.full_like(q.cuda(), 9.0)
    c.attend(q.cuda(), table, ints(vis), max_visible=L, out=out)
    c.sync()
    check(out, q, oracle.quantise(k.float().numpy()), oracle.quantise(v.float().numpy()), vis, dtype)
    assert torch.equal(out, c.attend(q.cuda(), table, ints(vis), max_visible=L))
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,n,group,L", [(64, 3, 1, 95), (128, 2, 4, 1500), (96, 34, 3, 333), (256, 1, 2, 64)])
def test_mask(dim, n, group, L, dtype):
    """Masks: random, a row that allows nothing, a row that allows one token;
    one row of it for all queries (stride 0), and an odd first byte."""
    g = np.random.default_rng(4)
    k, v = draw((2, L, 2, dim), dtype, 1), draw((2, L, 2, dim), dtype, 2)
    q = draw((2, n, 2 * group, dim), dtype, 3, 0.0)
    c, table = filled(k, v)
    kq, vq = oracle.quantise(k.float().numpy()), oracle.quantise(v.float().numpy())
    m = g.random((2, n, L + 3)) < 0.3
    m[0, 0] = False
    m[1, -1] = False
    m[1, -1, L // 2] = True
    vis = np.full((2, n), L)
    vis[0, -1] = L - 7
    part = torch.from_numpy(m).cuda()[:, :, 1:L + 1]
    out = c.attend(q.cuda(), table, ints(vis), mask=part)
    c.sync()
    check(out, q, kq, vq, vis, dtype, m[:, :, 1:L + 1])
    one = torch.from_numpy(m[:1, :1, 1:L + 1] | (np.arange(L) % 5 == 0)).cuda().expand(2, n, L)
    out = c.attend(q.cuda(), table, ints(vis), mask=one)
    c.sync()
    check(out, q, kq, vq, vis, dtype, one.cpu().numpy())
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_what_a_row_does_not_see(dim, dtype):
    """Blocks that are not finite: past every row's tokens, past one row's, and
    masked, they change nothing; in a key that a row sees they take the row, in
    a value the block's channels, of the rows that see them alone."""
    L, n = 200, 6
    k, v = draw((1, L, 1, dim), dtype, 1), draw((1, L, 1, dim), dtype, 2)
    k[0, 150:, 0, ::3] = float("nan")
    v[0, 150:, 0, ::5] = float("inf")
    v[0, 100, 0, 40] = float("nan")                 # block 1 of token 100
    k[0, 120, 0, 3] = float("-inf")
    v[0, 60, 0, 7] = float("inf")                   # masked for all but row 3
    q = draw((1, n, 2, dim), dtype, 3, 0.0)
    c, table = filled(k, v)
    kq, vq = oracle.quantise(k.float().numpy()), oracle.quantise(v.float().numpy())
    vis = np.array([[100, 101, 120, 100, 121, 150]])
    m = np.ones((1, n, L), bool)
    m[:, :, 60] = False
    m[0, 3, 60] = True
    m[0, 5, 100] = m[0, 5, 120] = False
    out = c.attend(q.cuda(), table, ints(vis), mask=torch.from_numpy(m).cuda())
    c.sync()
    got = np.isnan(out.float().cpu().numpy())[0]
    assert not got[0].any() and not got[5].any()
    assert got[1][:, 32:64].all() and got[1].sum() == 64 and got[3][:, :32].all() and got[3].sum() == 64
    assert got[2].sum() == 64 and got[4].all()
    check(out, q, kq, vq, vis, dtype, m)
    c.close()


@pytest.mark.parametrize("dim,n,group,heads,B", [(64, 130, 1, 2, 1), (128, 70, 3, 1, 2), (96, 64, 2, 1, 1), (64, 33, 8, 1, 1),
                                                 (128, 300, 1, 3, 1)])
def test_many_rows(dim, n, group, heads, B):
    """Many rows of unequal prefixes, some that see nothing or all; a key and
    values that are not finite at tokens that some of them see; a page outside
    the pool."""
    g = np.random.default_rng(7)
    L = 700
    k, v = draw((B, L, heads, dim), "bf16", 1), draw((B, L, heads, dim), "bf16", 2)
    q = draw((B, n, heads * group, dim), "bf16", 3, 0.0)
    for bad in (False, True):
        if bad:
            k[:, 600, :, 3] = float("nan")
            v[:, 500, :, 5] = float("inf")
            v[:, 501, :, dim - 1] = float("nan")
            k[0, 690:], v[0, 690:] = float("nan"), float("nan")
        c, table = filled(k, v)
        kq, vq = oracle.quantise(k.float().numpy()), oracle.quantise(v.float().numpy())
        vis = g.integers(0, L + 1, (B, n))
        vis[:, :3] = [[L, 0, 500]]
        vis[0, n // 2:] = np.minimum(vis[0, n // 2:], 500)
        if bad:
            vis[0] = np.minimum(vis[0], 690)
        out = c.attend(q.cuda(), table, ints(vis), max_visible=L)
        c.sync()
        check(out, q, kq, vq, vis, "bf16")
        assert torch.equal(out.nan_to_num(7.0), c.attend(q.cuda(), table, ints(vis), max_visible=L).nan_to_num(7.0))
        if not bad:
            broken = table.clone()
            broken[:, 4] = 1 << 30
            out = c.attend(q.cuda(), broken, ints(vis), max_visible=L)
            with pytest.raises(wf.WfError):
                c.sync()
            mask = np.ones((B, n, L), bool)
            mask[:, :, 256:320] = False
            check(out, q, kq, vq, vis, "bf16", mask)
        c.close()


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dim,n,group,heads,B,dtype", [(128, 256, 4, 8, 1, "bf16"), (128, 130, 4, 8, 2, "bf16"), (64, 515, 4, 8, 1, "bf16"),
                                                       (64, 512, 4, 8, 1, "fp32"), (96, 70, 1, 16, 8, "bf16")])
def test_rows_that_fill_the_chip(dim, n, group, heads, B, dtype, masked):
    """Enough rows for a workgroup to take two tiles of them: unequal prefixes,
    values that are not finite or far apart in size, a mask."""
    g = np.random.default_rng(13)
    L = 75
    k, v = draw((B, L, heads, dim), dtype, 1), draw((B, L, heads, dim), dtype, 2)
    q = draw((B, n, heads * group, dim), dtype, 3, 0.0)
    v[:, 10, 1] *= 2.0 ** 60
    v[:, 50, 2, 7] = float("nan")
    k[:, 51, 3, 1] = float("inf")
    k[:, 70:], v[:, 70:] = float("nan"), float("nan")
    c, table = filled(k, v)
    kq, vq = oracle.quantise(k.float().numpy()), oracle.quantise(v.float().numpy())
    vis = g.integers(0, 71, (B, n))
    vis[:, :2] = [[70, 0]]
    vis[:, n // 2:] = np.minimum(vis[:, n // 2:], 50)
    m = g.random((B, n, L)) < 0.4 if masked else None
    out = c.attend(q.cuda(), table, ints(vis), max_visible=L, mask=torch.from_numpy(m).cuda() if masked else None)
    c.sync()
    check(out, q, kq, vq, vis, dtype, m)
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,n,lens", [(260, 1, [8200]), (130, 2, [8193, 5000]), (64, 3, [8200, 0, 31, 2047, 1]),
                                          (45, 5, [8200, 0, 3000]), (88, 17, [8170])])
def test_a_few_more_than_compute_units(heads, n, lens, dtype):
    """Long calls whose workgroups would fill the compute units badly: 257 to
    320, or a half to five eighths of them (or of a part of them), are split."""
    B, L = len(lens), max(lens)
    k, v = draw((B, L, heads, 8), dtype, 1), draw((B, L, heads, 8), dtype, 2)
    q = draw((B, n, heads, 8), dtype, 3, 0.0)
    vis = [[max(0, x - i) for i in range(n)] for x in lens]
    c, table = filled(k, v, page=256)
    out = c.attend(q.cuda(), table, ints(vis), max_visible=L)
    c.sync()
    check(out, q, oracle.quantise(k.float().numpy()), oracle.quantise(v.float().numpy()), vis, dtype)
    c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,n,group,L", [(64, 1, 2, 300), (128, 3, 1, 600), (256, 1, 1, 90), (128, 400, 4, 70)])
def test_values_of_any_size(dim, n, group, L, dtype):
    """Values from 2^-100 to 2^100, in one channel or from token to token; the
    huge ones at tokens that other rows see or none sees change nothing else."""
    g = np.random.default_rng(11)
    heads = 8 if n > 100 else 2
    k, q = draw((1, L, heads, dim), dtype, 1), draw((1, n, heads * group, dim), dtype, 3, 0.0)
    for sizes in (2.0 ** g.integers(-100, 101, (L, heads, 1)), 2.0 ** -100 * np.ones((L, heads, 1)), 2.0 ** 100 * np.ones((L, heads, 1)),
                  2.0 ** g.integers(-100, 101, (1, heads, dim // 32)).repeat(32, -1).repeat(L, 0)):
        v = torch.from_numpy((g.standard_normal((L, heads, dim)) * sizes).astype(np.float32))[None].to(DTYPE[dtype])
        c, table = filled(k, v)
        kq, vq = oracle.quantise(k.float().numpy()), oracle.quantise(v.float().numpy())
        vis = g.integers(0, L + 1, (1, n))
        vis[0, -1] = L - 5
        out = c.attend(q.cuda(), table, ints(vis), max_visible=L)
        c.sync()
        check(out, q, kq, vq, vis, dtype)
        c.close()


def test_last_bits_of_fp32_queries_count():
    """A score of 1 that is the difference of two channels' 2^18: it needs the
    24 bits of the query, and the kernel's parts carry them."""
    k = torch.zeros((1, 2, 1, 64))
    k[0, 0, 0, :2] = 1.0
    v = torch.zeros((1, 2, 1, 64))
    v[0, 0] = 1.0
    q = torch.zeros((1, 1, 1, 64))
    q[..., 0], q[..., 1] = 2.0 ** 18, -(2.0 ** 18 - 1.0)
    c, table = filled(k, v)
    out = c.attend(q.cuda(), table, ints([[2]]), scale=1.0)
    assert abs(float(out[0, 0, 0, 0]) - 1 / (1 + np.exp(-1.0))) < 1e-6
    c.close()


def test_far_apart_scores():
    """Scores thousands apart, rising and falling along the tokens, in every
    split: the largest alone counts, and nothing overflows."""
    L = 3001
    for order in (1, -1):
        k = torch.ones((1, L, 1, 64)) * torch.arange(L)[None, :, None, None].float() / 100.0
        k = k if order == 1 else k.flip(1)
        v = torch.zeros((1, L, 1, 64))
        v[0, :, 0, :] = torch.arange(L)[:, None] % 7
        q = torch.full((1, 2, 1, 64), 30.0)
        q[0, 1] = -30.0
        c, table = filled(k, v)
        kq, vq = oracle.quantise(k.numpy()), oracle.quantise(v.numpy())
        out = c.attend(q.cuda(), table, ints([[L, L]]))
        c.sync()
        check(out, q, kq, vq, [[L, L]], "fp32")
        c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_views_streams_and_graphs(dtype):
    """Queries and outputs as views of wider arrays at odd addresses, calls on
    a stream of their own, and a captured step replayed between other work."""
    B, n, L, dim = 2, 3, 400, 128
    k, v = draw((B, L + 8, 2, dim), dtype, 1), draw((B, L + 8, 2, dim), dtype, 2)
    c, table = filled(k[:, :L], v[:, :L])
    table = torch.cat([table, ints([[0], [0]])], 1)   # unused columns
    q = draw((B, n, 4, dim), dtype, 3, 0.0)
    wide = torch.full((B, 4, n, 2 * dim + 1), 5.0, dtype=DTYPE[dtype], device="cuda")
    qv = wide[..., 1:dim + 1].transpose(1, 2)
    ov = wide[..., dim + 1:].transpose(1, 2)
    qv.copy_(q.cuda())
    vis = ints([[L, 7, 0], [L - 1, L, 350]])
    want = c.attend(q.cuda(), table, vis, max_visible=L)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.attend(qv, table, vis, max_visible=L, out=ov, stream=s)
    c.sync(s)
    assert torch.equal(ov, want) and (wide[..., 0] == 5).all() and torch.equal(qv, q.cuda())
    # a step: write one token, attend; replayed with other inputs in place
    first, kn, vn = ints([L, L]), k[:, L:L + 1].cuda(), v[:, L:L + 1].cuda()
    qs, out, vis = q.cuda(), torch.empty_like(want), ints([[L + 1, 7, 0], [L + 1, L, 350]])
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        c.write(kn, vn, table, first)
        c.attend(qs, table, vis, max_visible=L + 8, out=out)
    for t in range(1, 5):
        kn.copy_(k[:, L + t:L + t + 1])
        vn.copy_(v[:, L + t:L + t + 1])
        first.fill_(L)
        qs.mul_(0.5)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        c2, t2 = filled(torch.cat([k[:, :L], k[:, L + t:L + t + 1]], 1), torch.cat([v[:, :L], v[:, L + t:L + t + 1]], 1))
        want = c2.attend(qs, torch.cat([t2, ints([[0], [0]])], 1), vis, max_visible=L + 8)
        assert torch.equal(out, want), t
        c2.close()
    c.close()


# ---- what is refused, and what the kernels find ------------------------------------


def test_errors_found_by_the_kernels():
    k = draw((1, 70, 1, 64), "fp32", 1)
    c, table = filled(k, k, page=32)
    ref = c.read(table, ints([0]), 70)[0].clone()
    q = draw((1, 1, 1, 64), "fp32", 2).cuda()

    def raises(code):
        with pytest.raises(wf.WfError) as e:
            c.sync()
        assert e.value.code == code
        c.sync()                                    # cleared

    for first in (95, -1):                          # token 96, token -1
        c.write(k[:, :2].cuda(), k[:, :2].cuda(), table, ints([first]))
        raises(wf.WF_E_CAPACITY)
    assert torch.equal(c.read(table, ints([95]), 1)[0][0, 0], ref.new_tensor(oracle.quantise(k[0, 0].numpy())))
    c.write(k.cuda(), k.cuda(), table, ints([0]))
    got = c.read(table, ints([68]), 40)[0]
    raises(wf.WF_E_CAPACITY)
    assert torch.equal(got[:, :2], ref[:, 68:]) and (got[:, 28:] == 0).all()
    broken = table.clone()
    broken[0, 1] = 10 ** 6
    got = c.read(broken, ints([0]), 70)[0]
    raises(wf.WF_E_INVALID)
    assert torch.equal(got[:, :32], ref[:, :32]) and (got[:, 32:64] == 0).all() and torch.equal(got[:, 64:], ref[:, 64:])
    broken[0, 1] = -1
    c.write(k.cuda(), k.cuda(), broken, ints([0]))
    raises(wf.WF_E_INVALID)
    out = c.attend(q, broken, ints([[70]]))
    raises(wf.WF_E_INVALID)
    mask = torch.ones((1, 1, 70), dtype=torch.bool, device="cuda")
    mask[:, :, 32:64] = False
    assert torch.equal(out, c.attend(q, table, ints([[70]]), mask=mask, max_visible=70))
    out = c.attend(q, table, ints([[70]]), max_visible=50)
    raises(wf.WF_E_CAPACITY)
    assert torch.equal(out, c.attend(q, table, ints([[50]]), max_visible=50))
    c.close()


def test_refusals():
    c = wf.Cache(2, 64, 4, page=32)
    k = torch.zeros((1, 3, 2, 64), device="cuda")
    q = torch.zeros((1, 3, 4, 64), device="cuda")
    table, first, vis = ints([[0, 1]]), ints([0]), ints([[1, 2, 3]])
    for bad in ((k.half(), k.half()), (k, k.bfloat16()), (k[..., :32], k[..., :32]), (k.cpu(), k.cpu()), (k[:, :, :1], k[:, :, :1]),
                (k.transpose(2, 3).contiguous().transpose(2, 3), k), (k[0], k[0])):
        with pytest.raises(ValueError):
            c.write(*bad, table, first)
    for t, f, n in ((table.long(), first, None), (table, ints([0, 1]), None), (table, first, ints([[1]])), (table[0], first, None)):
        with pytest.raises(ValueError):
            c.write(k, k, t, f, counts=n)
        with pytest.raises((ValueError, IndexError)):
            c.read(t, f, 3, counts=n)
    for kw in (dict(scale=0.0), dict(scale=float("nan")), dict(scale=-1.0), dict(max_visible=65), dict(max_visible=-1)):
        with pytest.raises(wf.WfError) as e:
            c.attend(q, table, vis, **kw)
        assert e.value.code == wf.WF_E_INVALID
    with pytest.raises(wf.WfError):
        c.attend(q[:, :, :3], table, vis)
    for m in (torch.ones((1, 3, 8), device="cuda"), torch.ones((1, 2, 8), dtype=torch.bool, device="cuda")):
        with pytest.raises(ValueError):
            c.attend(q, table, vis, mask=m)
    with pytest.raises(ValueError):
        c.attend(q, table, vis[:, :2])
    # nothing to do is no error, and an empty row set writes nothing
    c.write(k[:, :0], k[:, :0], table, first)
    assert c.attend(q[:, :0], table, vis[:, :0].contiguous()).shape == (1, 0, 4, 64)
    assert (c.attend(q + 1, table, 0 * vis, max_visible=0) == 0).all()
    c.sync()
    c.close()


def test_a_pool_that_does_not_fit():
    with pytest.raises(wf.WfError) as e:
        wf.Cache(8, 128, 1 << 22, page=1024)        # 4.7 TB
    assert e.value.code == wf.WF_E_NOMEM
    # and nothing of it is left for the calls that follow
    k = draw((1, 40, 2, 64), "fp32", 1)
    c, table = filled(k, k, page=32)
    assert torch.equal(c.read(table, ints([0]), 40)[0][0].cpu(), torch.from_numpy(oracle.quantise(k[0].numpy())).float())
    c.sync()
    c.close()


def test_a_launch_that_is_too_large():
    c = wf.Cache(1, 8, 1)
    B = 1 << 23                                     # workgroups of 512 threads
    q = torch.zeros((B, 1, 1, 8), dtype=torch.bfloat16, device="cuda")
    table, visible = torch.empty((B, 0), dtype=torch.int32, device="cuda"), torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    with pytest.raises(wf.WfError) as e:
        c.attend(q, table, visible)
    assert e.value.code == wf.WF_E_UNSUPPORTED
    many = q.expand(B, 40, 1, 8)                    # which may reach into three records
    with pytest.raises(wf.WfError) as e:
        c.write(many, many, visible, visible[:, 0].contiguous())
    assert e.value.code == wf.WF_E_UNSUPPORTED
    half = slice(0, B // 2)
    assert (c.attend(q[half] + 1, table[half], visible[half]) == 0).all()
    c.sync()
    c.close()
