"""Rows that the windowed and the shared attention can get wrong, as in
test_cache_rows_gpu.py: the tokens that count are in either run.  u = 2^-24."""
import numpy as np
import pytest

import cache_precision as cp
from oracle import cache as oracle
from paper_2607_19082_amd import wf
from test_cache_gpu import DTYPE, U, draw, filled, ints
from test_cache_runs_gpu import behind

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wf.lib()  # fails loudly when the library is missing
    torch.cuda.set_device(0)


class Window:
    """Tokens of one sequence, of which rows see the last `own` and the first P."""

    def __init__(self, k, v, P, between=37):
        gap = draw((1, between) + k.shape[2:], "fp32", 77).to(k.dtype)      # that no row sees
        self.P, self.L = P, k.shape[1] + between
        self.c, self.table = filled(*(torch.cat([x[:, :P], gap, x[:, P:]], 1) for x in (k, v)))

    def attend(self, q, **kw):
        n = q.shape[1]
        return self.c.attend_window(q.cuda(), self.table, ints([[self.L] * n]), self.L - self.P - 37, self.P, max_visible=self.L, **kw)


class Shared:
    """The first P tokens as a prefix, the others as the own ones of copies of the
    sequence: many with a row or two each (whose rows are taken together over the
    prefix), or one with all."""

    def __init__(self, k, v, P, copies):
        self.P, self.L, self.copies = P, k.shape[1] - P, copies
        self.c, self.prefix, self.table = behind(k[0, :P], v[0, :P], *(x[:, P:].expand(copies, -1, -1, -1) for x in (k, v)))

    def attend(self, q, **kw):
        """Rows [1][n], dealt to the copies."""
        n, each = q.shape[1], -(-q.shape[1] // self.copies)
        rows = q[:, np.arange(each * self.copies) % n].reshape(self.copies, each, *q.shape[2:])
        fill = lambda x: torch.full((self.copies, each), x, dtype=torch.int32, device="cuda")  # noqa: E731
        out = self.c.attend_shared(rows.cuda(), self.prefix, fill(self.P), self.table, fill(self.L), max_prefix=self.P, max_visible=self.L, **kw)
        return out.reshape(1, -1, *q.shape[2:])[:, :n]


FORMS = {"window": Window, "together": lambda k, v, P: Shared(k, v, P, 16), "apart": lambda k, v, P: Shared(k, v, P, 1)}


@pytest.fixture(params=list(FORMS))
def form(request):
    return FORMS[request.param]


def rows_of(f, q, dtype, **kw):
    out = f.attend(q.to(DTYPE[dtype]), **kw)[0]
    f.c.sync()
    return out.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,L,P,at", [(64, 288, 100, 0), (128, 288, 100, 287), (256, 100, 64, 70), (64, 9001, 8000, 5), (128, 9001, 33, 9000),
                                        (128, 5, 3, 1)])
def test_small_probabilities_count(form, dim, L, P, at, dtype):
    """One token, in either run, holds nearly all of a row's weight and the value
    0: the outputs are the others' alone.  Bars as there."""
    g = np.random.default_rng(L + at)
    far = (4, 8, 16, 20, 24, 40, 70)
    k, v = torch.zeros((1, L, 1, dim)), torch.from_numpy(g.choice([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], (1, L, 1, dim))).float()
    k[0, :, 0, 0] = -1.0
    k[0, at] = v[0, at] = 0.0
    q = torch.zeros((1, len(far), 1, dim))
    q[0, :, 0, 0] = torch.tensor(far, dtype=torch.float32)
    f = form(k, v, P)
    out = rows_of(f, q, dtype, scale=1.0)[:, 0]
    for i, d in enumerate(far):
        p = np.exp(-float(d))
        ref = p * v[0, :, 0].double().numpy().sum(0) / (1 + p * (L - 1))
        tol = ref * (4 * (d + 4) + 2 * (L + 64)) * U
        if dtype == "bf16":
            tol = tol + ref * (2.0 ** -15 + 2.0 ** -8)
        assert (np.abs(out[i] - ref) <= tol).all(), (d, float((np.abs(out[i] - ref) / ref).max()))
    f.c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,L,P", [(64, 90, 50), (128, 700, 64), (256, 300, 100), (128, 9001, 8500)])
def test_large_scores(form, dim, L, P, dtype):
    """Finite scores from 2^20 to 2^100: a row is the mean of the values at its
    largest score, which are in both runs."""
    g = np.random.default_rng(L + dim)
    k, v = torch.zeros((1, L, 1, dim)), draw((1, L, 1, dim), dtype, 2).float()
    x = g.integers(-4, 5, L)
    x[[1, P - 1, L - 1]], x[[0, P, L - 2]] = 6, -6
    k[0, :, 0, 0] = torch.from_numpy(x).float()
    powers = np.concatenate([np.arange(20, 36), [40, 60, 100]])
    q = torch.zeros((1, 2 * len(powers), 1, dim))
    q[0, :, 0, 0] = torch.from_numpy(np.ldexp(g.uniform(1, 2, 2 * len(powers)), np.repeat(powers, 2)) * np.tile([1, -1], len(powers)))
    f = form(k.to(DTYPE[dtype]), v.to(DTYPE[dtype]), P)
    vq = oracle.quantise(v.to(DTYPE[dtype]).float().numpy())[0, :, 0]
    for scale in (1.0, 0.1):
        out = rows_of(f, q, dtype, scale=scale)[:, 0]
        for i in range(q.shape[1]):
            top = x == (6 if i % 2 == 0 else -6)
            ref, mag = vq[top].mean(0), np.abs(vq[top]).mean(0)
            tol = mag * 2 * (L + 64) * U
            if dtype == "bf16":
                tol = tol + mag * 2.0 ** -15 + np.abs(ref) * 2.0 ** -8
            assert (np.abs(out[i] - ref) <= tol).all(), (scale, i, powers[i // 2])
    f.c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,L,P,half", [(64, 40, 20, 20), (128, 700, 400, 500), (256, 300, 40, 20), (64, 9001, 4000, 4000)])
def test_scores_of_minus_infinity(form, dim, L, P, half, dtype):
    """Rows whose scores are all -infinity are NaN (0 / 0); tokens at -infinity, in
    one run or the other, have no part beside finite ones."""
    k, v = torch.zeros((1, L, 1, dim)), draw((1, L, 1, dim), dtype, 2)
    k[0, :, 0, 0] = -6.0
    k[0, half:, 0, 1] = -4.0
    k[0, :half, 0, 2] = -4.0
    q = torch.zeros((1, 4, 1, dim))
    q[0, 0, 0, :2] = torch.tensor([float("inf"), 1.0])     # -infinity throughout
    q[0, 1, 0, 1] = 3e38                                   # finite products below the range in the later part,
    q[0, 2, 0, 2] = 3e38                                   # in the earlier,
    q[0, 3, 0, 0] = 1.0                                    # and nowhere
    f = form(k.to(DTYPE[dtype]), v, P)
    out = rows_of(f, q, dtype, scale=1.0)[:, 0]
    vq = oracle.quantise(v.float().numpy())[0, :, 0]
    assert np.isnan(out[0]).all()
    for i, see in ((1, slice(0, half)), (2, slice(half, L)), (3, slice(0, L))):
        ref, mag = vq[see].mean(0), np.abs(vq[see]).mean(0)
        tol = mag * 2 * (L + 64) * U + (mag * 2.0 ** -15 + np.abs(ref) * 2.0 ** -8 if dtype == "bf16" else 0)
        assert (np.abs(out[i] - ref) <= tol).all(), i
    f.c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,tokens,P", [(64, 4, 2), (128, 3, 1), (256, 2, 1)])
def test_bits_of_a_probability(form, dim, tokens, P, dtype):
    """24 bits in fp32 calls and 16 in bf16 ones, by the bars of
    cache_precision.py: each row sees few tokens, of both runs."""
    q, k, v, _ = cp.case(dtype, dim, tokens, tokens)
    ref, mag, _ = oracle.attend(q, k, v, [tokens] * len(q), None, 1.0)
    f = form(*(torch.from_numpy(x)[None].to(DTYPE[dtype]) for x in (k, v)), P)
    got, bar = cp.misses(dtype, rows_of(f, torch.from_numpy(q)[None], dtype, scale=1.0), ref, mag)
    assert got <= bar, (got / U, bar / U)
    f.c.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,L,group", [(64, 300, 2), (128, 3000, 4), (256, 500, 1)])
def test_bits_do_not_depend_on_what_a_row_does_not_see(dim, L, group, dtype):
    """A row's bits stay, whatever lies between its window and the first tokens, or
    past what it sees of the prefix, where other rows of the call see it too."""
    n, window, sinks = 5, L // 4, 7
    k, v = draw((1, L, 1, dim), dtype, 1), draw((1, L, 1, dim), dtype, 2)
    q = draw((1, n, group, dim), dtype, 3, 0.0)
    hidden = slice(sinks, L - window)
    first = {}
    for what in ("as drawn", "large keys", "large values", "tiny values", "nan", "inf"):
        kw, vw = k.clone(), v.clone()
        if what == "large keys":
            kw[:, hidden] *= 64
        elif what == "large values":
            vw[:, hidden] *= 2.0 ** 60
        elif what == "tiny values":
            vw[:, hidden] *= 2.0 ** -60
        elif what == "nan":
            kw[:, hidden], vw[:, hidden] = float("nan"), float("nan")
        elif what == "inf":
            vw[:, hidden, :, ::40] = float("inf")
        c, table = filled(kw, vw)
        x = q.to(DTYPE[dtype]).cuda()
        # rows 3 and 4 see less of the sequence, and so hidden tokens
        got = {"window": c.attend_window(x, table, ints([[L, L, L, L - 50, L // 2]]), window, sinks, max_visible=L)[:, :3]}
        # as a prefix: rows 0 to 2 of every sequence see its first tokens alone
        for B in (1, 20):
            own = table[:, :2].expand(B, 2).contiguous()
            pvis = ints([[sinks, sinks, 3, L, L - window]] * B)
            got[B] = c.attend_shared(x.expand(B, -1, -1, -1).contiguous(), table[0], pvis, own, ints([[sinks, 5, 1, 0, 64]] * B),
                                     max_prefix=L, max_visible=64)[:, :3]
        c.sync()
        for name, out in got.items():
            assert torch.equal(out, first.setdefault(name, out)), (what, name)
        c.close()


def test_pool_beyond_4_gib():
    """Pages whose bytes lie past 2^32 in the pool."""
    heads, dim, page = 8, 256, 1024
    pages = (1 << 32) // (page * heads * dim * 17 // 16) + 8
    c = wf.Cache(heads, dim, pages, page=page)
    k, v = draw((1, 80, heads, dim), "bf16", 1), draw((1, 80, heads, dim), "bf16", 2)
    q = draw((6, 1, heads, dim), "bf16", 3, 0.0)
    prefix, table = ints([pages - 1]), ints([[pages - 2]] * 6)
    c.write(k[:, :40].cuda(), v[:, :40].cuda(), prefix[None], ints([0]))
    c.write(k[:, 40:].cuda(), v[:, 40:].cuda(), table[:1], ints([0]))
    both = ints([[pages - 3]])
    c.write(k.cuda(), v.cuda(), both, ints([0]))
    some = ints([[40]] * 6)
    out = c.attend_shared(q.cuda(), prefix, some, table, some, max_prefix=40, max_visible=40)
    last = c.attend_window(q.cuda(), both.expand(6, 1).contiguous(), ints([[80]] * 6), 30, 5, max_visible=80)
    c.sync()
    from test_cache_gpu import check
    kq, vq = (np.broadcast_to(oracle.quantise(x.float().numpy()), (6,) + x.shape[1:]) for x in (k, v))
    check(out, q, kq, vq, [[80]] * 6, "bf16")
    j = np.arange(80)
    check(last, q, kq, vq, [[80]] * 6, "bf16", np.broadcast_to((j >= 50) | (j < 5), (6, 1, 80)))
    c.close()
