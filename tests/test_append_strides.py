"""Token strides that the binding takes from tensors: rows that share memory are refused before the
library is called, which reads a stride of 0 as dense rows. On the host."""
import pytest
import torch

from paper_2602_01519_amd import pic


def closed_store():
    """A store without a handle: a call that reaches the library fails there with 'store is NULL'."""
    s = pic.Store.__new__(pic.Store)
    s.handle = None
    return s


def rows(n=50, heads=2, width=64):
    return torch.zeros(n, heads, width, dtype=torch.bfloat16)


def expanded(n=50, heads=2, width=64):
    return torch.zeros(1, heads, width, dtype=torch.bfloat16).expand(n, heads, width)


def append(**kw):
    with pytest.raises(pic.PicError) as e:
        closed_store().append([1], [0, 50], **{**dict(k=rows(), v=rows()), **kw})
    assert e.value.status == pic.ERR_INVALID
    return str(e.value)


@pytest.mark.parametrize("bad", [expanded(), expanded(heads=1), rows().as_strided((50, 2, 64), (64, 64, 1)),
                                 rows().as_strided((50, 2, 64), (127, 64, 1))], ids=["expanded", "one-head", "half", "short"])
@pytest.mark.parametrize("which", ["k", "v", "q", "q_out"])
def test_rows_that_share_memory(which, bad):
    kw = dict(q=rows(), q_out=rows()) if which.startswith("q") else {}
    assert "store is NULL" not in append(**{**kw, which: bad})


def test_rows_of_their_own_reach_the_library():
    wide = torch.zeros(50, 7, 64, dtype=torch.bfloat16)
    for kw in ({}, dict(q=rows(), q_out=rows()), dict(k=wide[:, 1:3], v=wide[:, 4:6]), dict(k=rows().data_ptr(), v=rows())):
        assert "store is NULL" in append(**kw)


@pytest.mark.parametrize("x,want", [
    (None, 0), (rows(), 128), (torch.zeros(9, 5, 64)[:, 1:3], 320), (torch.zeros(1, 2, 64), 0), (torch.zeros(0, 2, 64), 0),
    (torch.zeros(1, 2, 64).expand(1, 2, 64), 0), (torch.zeros(9, 1, 64), 64), (torch.zeros(9, 130)[:, :128].unflatten(1, (2, 64)), 130)])
def test_strides(x, want):
    assert pic._token_stride(x) == want
