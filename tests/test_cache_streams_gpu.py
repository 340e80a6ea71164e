"""The 4-bit cache's calls on a stream that is given: their memory is not
another stream's."""
import numpy as np
import pytest

from oracle import cache as oracle
from paper_2607_19082_amd import wf
from test_cache_gpu import draw, filled, ints

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wf.lib()  # fails loudly when the library is missing
    torch.cuda.set_device(0)


@pytest.fixture(scope="module")
def busy():
    """Some 10 ms of work on the current stream."""
    a = torch.zeros((8192, 8192), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(a)

    def work():
        for _ in range(8):
            torch.mm(a, a, out=out)

    work()
    torch.cuda.synchronize()
    return work


def test_outputs_are_not_memory_still_in_use(busy):
    """A tensor let go of by the current stream, which has yet to read it, is
    not what a call on another stream writes to."""
    k, v = draw((1, 40, 1, 64), "fp32", 1), draw((1, 40, 1, 64), "fp32", 2)
    c, table = filled(k, v)
    want = oracle.quantise(k.numpy()).astype(np.float32)
    first, vis, q = ints([0]), ints([[40] * 40]), draw((1, 40, 1, 64), "fp32", 3).cuda()
    out = c.attend(q, table, vis)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for call in (lambda: c.read(table, first, 40, stream=s)[0], lambda: c.attend(q, table, vis, stream=s)):
        x = [torch.full((1, 40, 1, 64), 5.0, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        busy()
        y = [t.clone() for t in x]
        del x
        got = call()
        c.sync(s)
        torch.cuda.synchronize()
        assert all((t == 5).all() for t in y)
        assert np.array_equal(got.cpu().numpy(), want) or torch.equal(got, out)
    c.close()


def test_inputs_are_kept_for_the_call(busy):
    """Inputs that are let go of right after a call on a busy stream are not
    given away before it has run."""
    L, n = 40, 7
    k, v = draw((1, L, 1, 64), "fp32", 1), draw((1, L, 1, 64), "fp32", 2)
    c, table = filled(k, v)
    q, vis = draw((1, n, 1, 64), "fp32", 3).cuda(), ints([[L] * n])
    mask = torch.ones((1, n, L), dtype=torch.bool, device="cuda")
    mask[:, :, ::3] = False
    want = c.attend(q, table, vis, mask=mask)
    s = torch.cuda.Stream()
    args = [q.clone(), table.clone(), vis.clone(), mask.clone()]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        busy()
    out = c.attend(args[0], args[1], args[2], mask=args[3], stream=s)
    shapes = [(t.shape, t.dtype) for t in args]
    del args
    over = [torch.zeros(shape, dtype=dtype, device="cuda") for shape, dtype in shapes * 3]
    c.sync(s)
    assert torch.equal(out, want)
    args = [k.cuda() + 1, v.cuda() + 1, table.clone(), ints([0]), ints([L])]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        busy()
    c.write(args[0], args[1], args[2], args[3], counts=args[4], stream=s)
    shapes = [(t.shape, t.dtype) for t in args]
    del args
    over += [torch.zeros(shape, dtype=dtype, device="cuda") for shape, dtype in shapes * 3]
    c.sync(s)
    gk, gv = c.read(table, ints([0]), L)
    for got, x in ((gk, k), (gv, v)):
        assert np.array_equal(got.cpu().numpy(), oracle.quantise((x + 1).numpy()).astype(np.float32))
    c.close()
