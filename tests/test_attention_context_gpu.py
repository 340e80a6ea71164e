"""The attention context example: encoder and decoder agree bit for bit, and
its contexts are those of 64 bits on the values that its cache holds.

Bar of the contexts, as for the attention alone (tests/test_cache_gpu.py): bf16
outputs are rounded to 2^-8, and their probabilities are held to 2^-16."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import cache as oracle
from paper_2607_19082_amd import inputs, wf

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wf.lib()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_context.py")
    spec = importlib.util.spec_from_file_location("attention_context", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("H,W,M,B,heads", [(6, 9, 192, 2, None), (5, 2, 192, 1, 1), (8, 12, 320, 1, None)])
def test_encoder_and_decoder_agree(example, H, W, M, B, heads):
    model = example.AttentionContext(H, W, M, B=B, heads=heads, page=32)
    psi = torch.from_numpy(inputs.make_psi(B, H, W, M)).cuda()
    y = 4 * torch.from_numpy(inputs.make_psi(B, H, W, M, seed=7)[..., :M].copy()).cuda()
    s, enc = model.encode(psi, y)
    dec = model.decode(psi, s)
    model.cache.sync()
    assert torch.equal(enc, dec)
    assert float((y - dec).abs().max()) <= 0.5 + 1e-4
    # the context of the last step's latents, from the values held
    k, v = (x.cpu().numpy() for x in model.cached())
    a, b = int(model.bounds[-2]), int(model.bounds[-1])
    p = model._ordered(psi)[:, a:b]
    q = (p @ model.wq).to(torch.bfloat16).view(B, b - a, model.q_heads, 64)
    got = model.cache.attend(q, model.table, torch.full((B, b - a), a, dtype=torch.int32, device="cuda"), max_visible=a)
    for i in range(B):
        ref, mag, big = oracle.attend(q[i].float().cpu().numpy(), k[i], v[i], [a] * (b - a))
        tol = mag * ((2 * 68 * big + 2 * (a + 64)) * 2.0 ** -24 + 2.0 ** -15) + np.abs(ref) * 2.0 ** -8
        assert (np.abs(got[i].float().cpu().numpy() - ref) <= tol).all()


def test_refuses_channels_off_the_head(example):
    with pytest.raises(ValueError):
        example.AttentionContext(4, 4, 100)
