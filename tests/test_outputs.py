"""Tensors that a caller gives to be written and that require a gradient: torch
does not see the write, so they would keep the gradient of what they held."""
import pytest
import torch

from paper_2607_19082_amd import wf


def call():
    """The calls' checks, for tensors of the CPU."""
    c = object.__new__(wf._TokenCalls)
    c._device = torch.empty(0).get_device()
    return c


def test_outputs_that_require_a_gradient():
    c, shape = call(), (1, 2, 3, 8)
    plain, leaf = torch.zeros(shape), torch.zeros(shape, requires_grad=True)
    made = leaf * 2
    assert c._output(plain, shape, torch.float32, "out") == c._rows(plain, shape, torch.float32, "out")
    for t in (leaf, made):
        with pytest.raises(ValueError, match="out: requires a gradient"):
            c._output(t, shape, torch.float32, "out")
        with torch.no_grad():
            before = t._version
            assert c._output(t, shape, torch.float32, "out") == c._rows(t, shape, torch.float32, "out")
            assert t._version == before + 1         # a graph that kept it for its backward pass finds that out
    with pytest.raises(ValueError, match="out: expected"):
        c._output(plain, (1, 2, 3, 16), torch.float32, "out")


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["norm", "norm keys", "attend", "window", "shared", "read"])
def test_calls(what):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    x = torch.randn((1, 2, 2, 64), device="cuda", requires_grad=True)
    q, other = x * 2, torch.zeros((1, 2, 2, 64), device="cuda")
    norm, cache = wf.HeadNorm(64), wf.Cache(2, 64, 2, page=32)
    cache.write(other, other, ints([[0]]), ints([0]))
    some, table = ints([[1, 2]]), ints([[0]])
    f = {"norm": lambda out: norm.apply(q, some, out=out), "norm keys": lambda out: norm.apply(other, some, k=q, out=(other, out)),
         "attend": lambda out: cache.attend(q, table, some, out=out), "window": lambda out: cache.attend_window(q, table, some, 1, out=out),
         "shared": lambda out: cache.attend_shared(q, table[0], some, table, some, out=out),
         "read": lambda out: cache.read(table, ints([0]), 2, out=(out, other))}[what]
    held = q.detach().clone()
    for out in (q, x):
        with pytest.raises(ValueError, match="requires a gradient"):
            f(out)
    assert torch.equal(q, held)                     # nothing was written
    y = (q * q).sum()
    with torch.no_grad():
        f(q)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    cache.sync()
    cache.close()
    norm.close()
