"""Shared-link and selected-block calls with tensors that start off 16 bytes: the bits of the same
call with aligned ones, nothing written around them."""
import numpy as np
import pytest
import torch

import link_model as L
from paper_2602_01519_amd import pic
from test_gpu_shared import SHAPES, Batch
from test_gpu_sparse import CHUNKS, LINKS, Case

pytestmark = pytest.mark.gpu


def off(x, fill=None):
    """A copy of x (or `fill` in its shape) one element into a buffer with a guard at either end."""
    if x is None:
        return None
    buf = torch.full((x.numel() + 2,), 9, dtype=x.dtype, device="cuda")
    y = buf[1:-1].view(x.shape)
    y.copy_(x) if fill is None else y.fill_(fill)
    assert y.data_ptr() % 16
    return y


def guarded(*ys):
    for y in ys:
        buf = torch.as_strided(y, (y.numel() + 2,), (1,), y.storage_offset() - 1)
        assert float(buf[0]) == 9 and float(buf[-1]) == 9


@pytest.mark.parametrize("shape", [s for s in SHAPES if not s[0].startswith("fp4")], ids=lambda s: s[0])
@pytest.mark.parametrize("q_len", [1, 6, 21])
def test_shared(shape, q_len):
    rng = np.random.default_rng(q_len)
    b = Batch(rng, *shape[1:], [3, 1], [[130, 20], [64]], [[20], [], [70], []], [q_len] * 4, own=[3, 0, 64, 5])
    want = b.call()
    b.check(*want)
    b.q, b.ko, b.vo = off(b.q), off(b.ko), off(b.vo)
    out, lse = off(want[0], 7), off(want[1], 3)
    b.call(out=out, lse=lse)
    torch.cuda.synchronize()
    same = torch.equal(out, want[0]), torch.equal(lse, want[1])
    assert same == (True, True)
    guarded(out, lse)
    with b.plan() as plan:
        b.run(plan, 0, out.fill_(7), lse.fill_(3))
        torch.cuda.synchronize()
    same = torch.equal(out, want[0]), torch.equal(lse, want[1])
    assert same == (True, True)
    guarded(out, lse)


@pytest.mark.parametrize("dtype", [pic.BF16, pic.F32])
@pytest.mark.parametrize("d,group", [(128, 4), (64, 3), (64, 8)])
@pytest.mark.parametrize("n", [3, 16])
def test_sparse(dtype, d, group, n):
    rng = np.random.default_rng(d + group + n)
    c = Case(rng, dtype, 2, d, group, CHUNKS, LINKS, [1, 2, 1, 3, 0, 1], own=[0, 70, 5, 0, 3, 200])
    want = c.call(n, 1, 1)
    c.check(want, n, 1, 1)
    c.q, c.ko, c.vo = off(c.q), off(c.ko), off(c.vo)
    bufs = tuple(off(x, f) for x, f in zip(want, (7, 3, -9)))
    c.call(n, 1, 1, bufs=bufs)
    torch.cuda.synchronize()
    same = [torch.equal(a, b) for a, b in zip(bufs, want)]
    assert same == [True] * 3
    guarded(*bufs)
