"""Rows that the 4-bit cache's attention can get wrong.  u = 2^-24."""
import numpy as np
import pytest

import cache_precision as cp
from oracle import cache as oracle
from paper_2607_19082_amd import wf
from test_cache_gpu import DTYPE, U, draw, filled, ints

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wf.lib()  # fails loudly when the library is missing
    torch.cuda.set_device(0)


def attend(c, q, table, vis, dtype, **kw):
    out = c.attend(q.to(DTYPE[dtype]).cuda(), table, ints(vis), **kw)
    c.sync()
    return out


# ---- probabilities far below the largest ------------------------------------------


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,L,at", [(64, 288, 0), (64, 288, 150), (128, 288, 287), (256, 100, 3), (64, 9001, 0), (128, 9001, 9000),
                                      (256, 9001, 4500), (128, 3, 1)])
def test_small_probabilities_count(dim, L, at, dtype):
    """One token holds nearly all of a row's weight and the value 0, so that the
    outputs are the others' alone, d nats below it.

    A score is one exact product, its power of two is off by 2 d u at most and
    its probability by a few u more; sums as in the other tests: |out - ref| <=
    A (4 (d + 4) + 2 (L + 64)) u, and bf16's 16 bits and rounding.  Each output
    has one sign, so A = |ref|."""
    g = np.random.default_rng(L + at)
    far = (4, 8, 16, 20, 24, 40, 70)
    k, v = torch.zeros((1, L, 1, dim)), torch.from_numpy(g.choice([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], (1, L, 1, dim))).float()
    k[0, :, 0, 0] = -1.0
    k[0, at] = v[0, at] = 0.0
    q = torch.zeros((1, len(far), 1, dim))
    q[0, :, 0, 0] = torch.tensor(far, dtype=torch.float32)
    c, table = filled(k, v)
    out = attend(c, q, table, [[L] * len(far)], dtype, scale=1.0)[0, :, 0].float().cpu().numpy().astype(np.float64)
    for i, d in enumerate(far):
        p = np.exp(-float(d))
        ref = p * v[0, :, 0].double().numpy().sum(0) / (1 + p * (L - 1))
        tol = ref * (4 * (d + 4) + 2 * (L + 64)) * U
        if dtype == "bf16":
            tol = tol + ref * (2.0 ** -15 + 2.0 ** -8)
        assert (np.abs(out[i] - ref) <= tol).all(), (d, float((np.abs(out[i] - ref) / ref).max()))
    c.close()


# ---- what other rows see -------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,L,group", [(64, 200, 2), (128, 3000, 4), (256, 500, 1), (128, 70, 8)])
def test_bits_do_not_depend_on_what_a_row_does_not_see(dim, L, group, dtype):
    """A row's bits stay, whatever lies at tokens that its mask or its prefix
    leaves out, where other rows of the call see them too: ordinary values,
    large keys, large or tiny values, blocks that are not finite, tokens never
    written (those that no row sees)."""
    g = np.random.default_rng(17)
    n = 5
    k, v = draw((1, L, 1, dim), dtype, 1), draw((1, L, 1, dim), dtype, 2)
    q = draw((1, n, group, dim), dtype, 3, 0.0)
    hidden = g.random(L) < 0.3
    hidden[0] = False
    hidden[L - 20:] = True
    # rows 0 to 2 never see the hidden tokens; rows 3 and 4 see those of them in `shown`
    for shown in (np.zeros(L, bool), hidden & (np.arange(L) < L - 20)):
        m = np.tile(~hidden, (1, n, 1))
        m[0, 3:] |= shown
        m[0, 1] &= g.random(L) < 0.5
        vis = [[L - 20, L - 20, L // 2, L - 20, L - 20]]
        first = None
        for what in ("as drawn", "large keys", "large values", "tiny values", "nan", "inf", "never written"):
            kw, vw = k.clone(), v.clone()
            h = torch.from_numpy(hidden)
            if what == "large keys":
                kw[:, h] *= 64
            elif what == "large values":
                vw[:, h] *= 2.0 ** 60
            elif what == "tiny values":
                vw[:, h] *= 2.0 ** -60
            elif what == "nan":
                kw[:, h], vw[:, h] = float("nan"), float("nan")
            elif what == "inf":
                vw[:, h, :, ::40] = float("inf")
            c, table = filled(kw, vw)
            if what == "never written":
                if shown.any():
                    c.close()
                    continue
                c.close()
                c = wf.Cache(1, dim, c.pages)
                for t in np.flatnonzero(~hidden):
                    c.write(k[:, t:t + 1].cuda(), v[:, t:t + 1].cuda(), table, ints([t]))
            out = attend(c, q, table, vis, dtype, mask=torch.from_numpy(m).cuda())[:, :3]
            first = out if first is None else first
            assert torch.equal(out, first), (what, bool(shown.any()))
            c.close()


# ---- large scores -----------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,L", [(64, 90), (128, 700), (256, 300), (64, 9001), (128, 9001)])
def test_large_scores(dim, L, dtype):
    """Finite scores from 2^20 to 2^100 with gaps of thousands between unequal
    ones: a row is the mean of the values at its largest score, which are held
    by several tokens of several waves and splits."""
    g = np.random.default_rng(L + dim)
    k, v = torch.zeros((1, L, 1, dim)), draw((1, L, 1, dim), dtype, 2).float()
    x = g.integers(-4, 5, L)
    x[g.random(L) < 0.02] = 6
    x[g.random(L) < 0.02] = -6
    x[[1, L - 1]], x[[0, L - 2]] = 6, -6
    k[0, :, 0, 0] = torch.from_numpy(x).float()
    powers = np.concatenate([np.arange(20, 36), [40, 60, 100]])
    q = torch.zeros((1, 2 * len(powers), 1, dim))
    q[0, :, 0, 0] = torch.from_numpy(np.ldexp(g.uniform(1, 2, 2 * len(powers)), np.repeat(powers, 2)) * np.tile([1, -1], len(powers)))
    q = q.to(DTYPE[dtype])
    c, table = filled(k.to(DTYPE[dtype]), v.to(DTYPE[dtype]))
    vq = oracle.quantise(v.to(DTYPE[dtype]).float().numpy())[0, :, 0]
    for scale in (1.0, 0.125, 0.1):
        out = attend(c, q, table, [[L] * q.shape[1]], dtype, scale=scale)[0, :, 0].float().cpu().numpy().astype(np.float64)
        for i in range(q.shape[1]):
            top = x == (6 if i % 2 == 0 else -6)
            ref, mag = vq[top].mean(0), np.abs(vq[top]).mean(0)
            tol = mag * 2 * (L + 64) * U
            if dtype == "bf16":
                tol = tol + mag * 2.0 ** -15 + np.abs(ref) * 2.0 ** -8
            assert (np.abs(out[i] - ref) <= tol).all(), (scale, i, powers[i // 2], out[i][:4], ref[:4])
    c.close()


# ---- scores that are infinite ---------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,L", [(64, 40), (128, 700), (256, 300), (64, 9001)])
def test_scores_of_minus_infinity(dim, L, dtype):
    """Rows that see tokens, all at -infinity, are NaN (0 / 0); tokens at
    -infinity beside finite ones have no part; rows that see nothing are zeros."""
    k, v = torch.zeros((1, L, 1, dim)), draw((1, L, 1, dim), dtype, 2)
    k[0, :, 0, 0] = -6.0
    k[0, L // 2:, 0, 1] = -4.0
    q = torch.zeros((1, 6, 1, dim))
    q[0, 0, 0, :2] = torch.tensor([float("inf"), 1.0])     # -infinity throughout
    q[0, 1, 0, :2] = torch.tensor([float("inf"), 1.0])     # one token of it
    q[0, 2, 0, 1] = 3e38                                   # finite products below the range in the later half
    q[0, 3] = q[0, 2]                                      # and no other tokens seen
    q[0, 4, 0, 0] = float("inf")                           # sees nothing
    q[0, 5, 0, 0] = 1.0
    c, table = filled(k.to(DTYPE[dtype]), v)
    m = np.ones((1, 6, L), bool)
    m[0, 1, np.arange(L) != L // 3] = False
    m[0, 3, :L // 2] = False
    m[0, 4] = False
    out = attend(c, q, table, [[L] * 6], dtype, mask=torch.from_numpy(m).cuda(), scale=1.0)[0, :, 0].float().cpu().numpy()
    nothing = attend(c, q, table, [[0] * 5 + [L]], dtype, max_visible=L)[0, :, 0].float().cpu().numpy()
    vq = oracle.quantise(v.float().numpy())[0, :, 0]
    for i, see in ((2, slice(0, L // 2)), (5, slice(0, L))):
        ref, mag = vq[see].mean(0), np.abs(vq[see]).mean(0)
        tol = mag * 2 * (L + 64) * U + (mag * 2.0 ** -15 + np.abs(ref) * 2.0 ** -8 if dtype == "bf16" else 0)
        assert (np.abs(out[i] - ref) <= tol).all(), i
    assert np.isnan(out[[0, 1, 3]]).all() and (out[4] == 0).all()
    assert (nothing[:5] == 0).all() and np.isfinite(nothing[5]).all()
    c.close()


# ---- the bits of a probability ----------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,L,sees", cp.CASES)
def test_bits_of_a_probability(dim, L, sees, dtype):
    """24 bits in fp32 calls and 16 in bf16 ones, by bars that fewer do not
    pass (derived in cache_precision.py, and shown on a model on the CPU)."""
    q, k, v, mask = cp.case(dtype, dim, L, sees)
    ref, mag, _ = oracle.attend(q, k, v, [L] * len(q), mask, 1.0)
    c, table = filled(*(torch.from_numpy(x)[None].to(DTYPE[dtype]) for x in (k, v)))
    out = attend(c, torch.from_numpy(q)[None], table, [[L] * len(q)], dtype, mask=torch.from_numpy(mask)[None].cuda(), scale=1.0)
    got, bar = cp.misses(dtype, out[0].float().cpu().numpy(), ref, mag)
    assert got <= bar, (got / U, bar / U)
    c.close()


# ---- counts that ctypes would cut down --------------------------------------------------


def test_counts_beyond_32_bits_are_refused():
    c, table = filled(torch.ones((1, 3, 1, 64)), torch.ones((1, 3, 1, 64)))
    q, vis = torch.ones((1, 1, 1, 64), device="cuda"), ints([[3]])
    for most in (1 << 32, (1 << 32) + 3, 3 - (1 << 32)):
        with pytest.raises(ValueError):
            c.attend(q, table, vis, max_visible=most)
    many = torch.ones((1, 1, 1, 64), device="cuda").expand(1, (1 << 32) + 1, 1, 64)
    with pytest.raises(ValueError):
        c.write(many, many, table, ints([0]))
    with pytest.raises(ValueError):
        c.read(table, ints([0]), (1 << 32) + 1, out=(many, many))
    assert (c.attend(q, table, vis, max_visible=3) == 1).all()
    c.close()
