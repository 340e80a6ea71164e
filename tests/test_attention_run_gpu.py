"""Head norms, the cache, and its windowed and shared attention together, as an
attention context model and a batch of requests run them.  Each call is held to
its own bar on what the call before it gave."""
import numpy as np
import pytest

from oracle import cache as oracle
from paper_2607_19082_amd import inputs, wf
from test_attention_context_gpu import example  # noqa: F401 (a fixture)
from test_cache_gpu import check, ints
from test_head_norm_gpu import close

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wf.lib()  # fails loudly when the library is missing
    torch.cuda.set_device(0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_requests_behind_a_prompt(dtype):
    """A prompt of 200 tokens, then three tokens each of five requests behind it:
    queries and keys are taken from a fused projection's output, normed and
    rotated in place, keys and values join the cache, and queries attend to the
    prompt and their own tokens.  The first request also runs by itself, its
    prompt in its own pages, with a window that holds everything and a short one."""
    B, P, n, hq, h, D, page = 5, 200, 3, 8, 2, 64, 32
    t = torch.float32 if dtype == "fp32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda").to(t)  # noqa: E731
    norm = wf.HeadNorm(D, base=500.0)
    gains = torch.rand((2, D), generator=g, device="cuda") + 0.5
    f = 500.0 ** (-np.arange(D // 2) / (D // 2))
    c = wf.Cache(h, D, 32, page=page)
    prefix, table, alone = ints(np.arange(7)), ints(7 + np.arange(B)[:, None]), ints([np.arange(20, 28)])

    def enter(fused, positions, table, first):
        """Norms and rotates a projection's queries and keys, writes, and checks both."""
        q, k, v = fused[:, :, :hq], fused[:, :, hq:hq + h], fused[:, :, hq + h:]
        before = fused.clone()
        norm.apply(q, positions, k=k, q_gain=gains[0], k_gain=gains[1], out=(q, k))
        for x, y, gain in ((before[:, :, :hq], q, gains[0]), (before[:, :, hq:hq + h], k, gains[1])):
            close(y, x, positions.cpu().numpy()[..., None], dtype, gain=gain.cpu().numpy(), eps=float(np.float32(1e-6)),
                  frequencies=f, rotated=D)
        assert torch.equal(before[:, :, hq + h:], v)
        c.write(k, v, table, first)
        got = c.read(table, first, k.shape[1])
        c.sync()
        for x, y in zip((k, v), got):
            assert np.array_equal(y.cpu().numpy(), oracle.quantise(x.float().cpu().numpy()).astype(np.float32))
        return q, got

    prompt = draw(1, P, hq + 2 * h, D)
    positions = torch.arange(P, dtype=torch.int32, device="cuda")[None]
    _, (pk, pv) = enter(prompt.clone(), positions, prefix[None], ints([0]))
    q0, _ = enter(prompt.clone(), positions, alone, ints([0]))
    # the prompt itself, in a window of 50 tokens and four first ones
    vis = positions + 1
    out = c.attend_window(q0, alone, vis, 50, 4, max_visible=P)
    j, v = np.arange(P), vis.cpu().numpy()[..., None]
    check(out, q0.cpu(), pk.cpu().numpy(), pv.cpu().numpy(), vis.cpu().numpy(), dtype, (j < v) & ((j >= v - 50) | (j < 4)))
    keys, values = [], []
    for step in range(n):
        fused = draw(B, 1, hq + 2 * h, D)
        at = torch.full((B, 1), P + step, dtype=torch.int32, device="cuda")
        q, (k, v) = enter(fused.clone(), at, table, ints([step] * B))
        keys.append(k)
        values.append(v)
        pvis, vis = ints([[P]] * B), ints([[step + 1]] * B)
        out = c.attend_shared(q, prefix, pvis, table, vis, max_prefix=P, max_visible=step + 1)
        c.sync()
        kk, vv = (torch.cat([x.expand(B, -1, -1, -1)] + y, 1).cpu().numpy() for x, y in ((pk, keys), (pv, values)))
        check(out, q.cpu(), kk, vv, [[P + step + 1]] * B, dtype)
        # the first request by itself
        q1, _ = enter(fused[:1].clone(), at[:1], alone, ints([P + step]))
        assert torch.equal(q1, q[:1])
        for window in (P + n, 40):
            vis = ints([[P + step + 1]])
            out = c.attend_window(q1, alone, vis, window, 7, max_visible=P + step + 1)
            c.sync()
            j = np.arange(P + step + 1)
            check(out, q1.cpu(), kk[:1], vv[:1], [[P + step + 1]], dtype, ((j >= P + step + 1 - window) | (j < 7))[None, None])
    c.close()
    norm.close()


@pytest.mark.parametrize("H,W,M,B,window,sinks", [(6, 9, 192, 2, 20, 3), (8, 12, 320, 1, 33, 0), (5, 2, 192, 1, 1, 0), (9, 16, 192, 1, None, 0)])
def test_encoder_and_decoder_agree(example, H, W, M, B, window, sinks):  # noqa: F811
    """With queries and keys rotated by row and column and a window, they see the
    same cache."""
    model = example.AttentionContext(H, W, M, B=B, page=32, placed=True, window=window, sinks=sinks)
    psi = torch.from_numpy(inputs.make_psi(B, H, W, M)).cuda()
    y = 4 * torch.from_numpy(inputs.make_psi(B, H, W, M, seed=7)[..., :M].copy()).cuda()
    s, enc = model.encode(psi, y)
    dec = model.decode(psi, s)
    model.cache.sync()
    assert torch.equal(enc, dec)
    assert float((y - dec).abs().max()) <= 0.5 + 1e-4
    # another place is another context: the rotation has a part in it, unless a
    # latent sees one other, whose weight is 1 whatever its score
    if window == 1:
        return
    plain = example.AttentionContext(H, W, M, B=B, page=32, window=window, sinks=sinks)
    assert not torch.equal(plain.encode(psi, y)[1], enc)


def test_search(example):  # noqa: F811
    """Each way's context is that of the coded latents and its own, from the values
    that the cache holds; rounding to the nearest has the least error."""
    H, W, M, C = 8, 12, 192, 5
    model = example.AttentionContext(H, W, M, page=32, placed=True, spare=16)
    psi = torch.from_numpy(inputs.make_psi(1, H, W, M)).cuda()
    y = 4 * torch.from_numpy(inputs.make_psi(1, H, W, M, seed=7)[..., :M].copy()).cuda()
    step, ahead = 10, 3
    error = model.search(psi, y, step, ahead, [-0.4, -0.2, 0.0, 0.2, 0.4])
    model.cache.sync()
    assert error.argmin() == 2 and torch.isfinite(error).all()
    start, a, b = (int(model.bounds[step + i]) for i in (0, ahead - 1, ahead))
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    pk, pv = model.cache.read(model.table, zero, start)
    k, v = model.cache.read(model.spare[:C][:, None].contiguous(), zero.expand(C).contiguous(), a - start)
    q = model._heads(model._ordered(psi)[:, a:b].expand(C, -1, -1), model.wq, model.q_heads, a)
    seen = [torch.full((C, b - a), x, dtype=torch.int32, device="cuda") for x in (start, a - start)]
    out = model.cache.attend_shared(q, model.table[0, :-(-start // 32)].contiguous(), seen[0], model.spare[:C][:, None].contiguous(), seen[1],
                                    max_prefix=start, max_visible=a - start)
    kk, vv = (torch.cat([x.expand(C, -1, -1, -1), z], 1).cpu().numpy() for x, z in ((pk, k), (pv, v)))
    check(out, q.cpu(), kk, vv, np.full((C, b - a), a), "bf16")
    # more ways than there are spare pages for
    with pytest.raises(ValueError):
        model.search(psi, y, step, 3, [0.0] * 17)
