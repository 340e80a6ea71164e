"""Head norms whose outputs are stored past the caches (32 MB and more), against
64 bits; the bar is test_head_norm_gpu.py's.  Inputs are made on the GPU, and
tokens here and there are compared."""
import numpy as np
import pytest

from paper_2607_19082_amd import wf
from test_head_norm_gpu import DTYPE, close

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

MOST = 32 << 20     # bytes of outputs that are stored through the caches


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wf.lib()  # fails loudly when the library is missing
    torch.cuda.set_device(0)


def rows(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda") * torch.exp2(4 * torch.randn(shape[:2] + (1, 1), generator=g, device="cuda"))
    return x.to(DTYPE[dtype])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("B,n,hq,hk,dim,rotated,axes", [
    (1, 14001, 5, 5, 64, 64, 2), (2, 7001, 11, 3, 64, 32, 1), (3, 2800, 6, 2, 256, 256, 1), (1, 5003, 7, 7, 256, 64, 2), (2, 4100, 32, 8, 128, 128, 2),
    (1, 20001, 17, 0, 56, 56, 1)])
def test_past_the_caches(B, n, hq, hk, dim, rotated, axes, pairs, dtype):
    """New outputs, then in place on views at odd addresses, with counts."""
    item = 4 if dtype == "fp32" else 2
    extra = -(-MOST // (B * n * (hq + hk) * dim * item))        # bf16 has more tokens for as many bytes
    n *= max(1, extra)
    assert B * n * (hq + hk) * dim * item > MOST
    wide = rows((B, n, hq + hk + 1, dim + 1), dtype, 1)
    q, k = wide[:, :, :hq, 1:], wide[:, :, hq:hq + hk, 1:] if hk else None
    g = torch.Generator(device="cuda").manual_seed(2)
    positions = torch.randint(-5000, 5001, (B, n) if axes == 1 else (B, n, 2), generator=g, device="cuda", dtype=torch.int32)
    gains = 1 + 0.5 * torch.randn((2, dim), generator=g, device="cuda")
    norm = wf.HeadNorm(dim, eps=1e-5, base=1000.0, rotated=rotated, axes=axes, pairs=pairs)
    each = rotated // (2 * axes)
    kw = dict(eps=float(np.float32(1e-5)), frequencies=1000.0 ** (-np.arange(each) / each), rotated=rotated, pairs=pairs)
    got = norm.apply(q, positions, k=k, q_gain=gains[0], k_gain=gains[1] if hk else None)
    got = got if hk else (got,)
    some = torch.tensor(sorted({0, 1, 2, 777, n // 2, n - 2, n - 1}))
    at = positions[:, some].cpu().numpy().reshape(B, len(some), axes)
    for x, y, gain in zip((q, k), got, gains):
        close(y[:, some], x[:, some], at, dtype, gain=gain.cpu().numpy(), **kw)
        # by itself, in parts that are stored through the caches: the same bits
        part = 1 + (MOST // item - 1) // (B * max(hq, hk) * dim) // 2
        for a in range(0, n, part):
            s = slice(a, min(n, a + part))
            assert torch.equal(norm.apply(x[:, s].contiguous(), positions[:, s].contiguous(), q_gain=gain), y[:, s])
    counts = torch.tensor([n - 5, 0, n // 3][:B], dtype=torch.int32, device="cuda")
    on = (torch.arange(n, device="cuda") < counts[:, None])[..., None, None]
    expect = wide.clone()
    expect[:, :, :hq, 1:] = torch.where(on, got[0], q)
    if hk:
        expect[:, :, hq:hq + hk, 1:] = torch.where(on, got[1], k)
    norm.apply(q, positions, k=k, q_gain=gains[0], k_gain=gains[1] if hk else None, counts=counts, out=(q, k) if hk else q)
    assert torch.equal(wide, expect)
    norm.close()
