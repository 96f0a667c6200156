"""Refusals of the 4-bit stores and the rotary positions: on the host, before any device work."""
import ctypes

import numpy as np
import pytest

import fp4_model as M
from paper_2602_01519_amd import pic


@pytest.mark.parametrize("desc", [
    dict(kind=pic.MLA, n_kv_heads=1, d_k=576, d_v=512), dict(d_k=96, d_v=96), dict(d_k=128, d_v=64),
    dict(d_k=32, d_v=32), dict(d_k=256, d_v=256)])
def test_shapes_without_a_4_bit_kernel(desc):
    d = pic.StoreDesc(**{**dict(kind=pic.GQA, dtype=pic.FP4, n_kv_heads=2, d_k=128, d_v=128, n_layers=0,
                                capacity_tokens=1024), **desc})
    h = ctypes.c_void_p(1)
    assert pic.lib().pic_store_create(ctypes.byref(d), ctypes.byref(h)) == pic.ERR_UNSUPPORTED
    assert not h.value and pic.last_error()


GOOD = dict(dtype=pic.BF16, layout=pic.ROPE_HALF, head_dim=128, rot_at=0, rot_dim=128)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=pic.FP4), pic.ERR_INVALID), (dict(layout=2), pic.ERR_INVALID),
    (dict(rot_dim=0), pic.ERR_INVALID), (dict(rot_dim=63), pic.ERR_INVALID),
    (dict(rot_at=2), pic.ERR_INVALID), (dict(rot_at=-2, rot_dim=64), pic.ERR_INVALID),
    (dict(rot_at=2 ** 31 - 1, rot_dim=64), pic.ERR_INVALID),
    (dict(head_dim=512, rot_dim=258), pic.ERR_UNSUPPORTED), (dict(head_dim=769), pic.ERR_UNSUPPORTED),
    (dict(theta=0.0), pic.ERR_INVALID), (dict(theta=float("nan")), pic.ERR_INVALID),
    (dict(magnitude=0.0), pic.ERR_INVALID), (dict(scaling=4), pic.ERR_INVALID),
    (dict(scaling=-1), pic.ERR_INVALID), (dict(scaling=pic.ROPE_LINEAR, factor=0.0), pic.ERR_INVALID),
    (dict(scaling=pic.ROPE_BANDED, factor=8.0), pic.ERR_INVALID),
    (dict(scaling=pic.ROPE_BANDED, factor=8.0, original_len=8192, band_low=4, band_high=4), pic.ERR_INVALID),
    (dict(scaling=pic.ROPE_YARN, factor=8.0, original_len=4096, turns_fast=1, turns_slow=32), pic.ERR_INVALID),
    (dict(scaling=pic.ROPE_YARN, factor=8.0, original_len=4096, turns_fast=32, turns_slow=1, theta=1.0),
     pic.ERR_INVALID)])
def test_rope_descriptions(bad, status):
    with pytest.raises(pic.PicError) as e:
        pic.Rope(**{**GOOD, **bad})
    assert e.value.status == status


def test_rope_calls():
    L = pic.lib()
    assert L.pic_rope_create(None, None) == pic.ERR_INVALID
    assert L.pic_rope_destroy(None) == pic.OK
    assert L.pic_rope_apply(None, 1, None, None, 1, 0, None) == pic.ERR_INVALID
    x = np.zeros(4096, np.int16)               # never read: every call here is refused
    a = x.ctypes.data
    with pic.Rope(**GOOD) as rope:
        rope.apply(0, None, [(None, None, 1, 0, 0)])            # nothing to do
        for n, pos, tensors in [
                (-1, a, [(a, a, 1, 0, 0)]), (1, None, [(a, a, 1, 0, 0)]), (1, a, []),
                (1, a, [(a, a, 1, 0, 0)] * 5), (1, a, [(None, a, 1, 0, 0)]), (1, a, [(a, None, 1, 0, 0)]),
                (1, a, [(a, a, 0, 0, 0)]), (1, a, [(a, a, 1025, 0, 0)]), (1, a, [(a, a, 2, 255, 0)]),
                (1, a, [(a, a + 4096, 2, 0, -1)]), (1, a, [(a, a, 1, 128, 256)]),
                (1, a, [(a + 1, a, 1, 0, 0)]), (1, a, [(a, a, 1, 0, 0), (a, None, 1, 0, 0)])]:
            with pytest.raises(pic.PicError) as e:
                rope.apply(n, pos, tensors)
            assert e.value.status == pic.ERR_INVALID, (n, tensors)
    with pytest.raises(pic.PicError):
        rope.apply(0, None, [(None, None, 1, 0, 0)])            # closed


def test_model_of_the_format():
    """The oracle's own pins: every code is kept, borders go to the even code, the scale rule."""
    x = np.concatenate([M.GRID, -M.GRID, M.GRID, M.GRID])[None]
    assert np.array_equal(M.stored(x), x)
    for top, want in [(6.0, 6.0), (6.75, 6.0), (6.96875, 6.0), (7.0, 8.0), (7.5, 8.0), (5.0, 4.0),
                      (3.5, 4.0), (3.25, 3.0), (np.inf, 6 * 2.0 ** 125), (2.0 ** -127, 2.0 ** -127),
                      (2.0 ** -129, 0.0)]:
        x = np.zeros((1, 32))
        x[0, 0] = top
        assert M.stored(x)[0, 0] == want, top
    x = np.zeros((1, 64))
    x[0, 40] = np.nan
    assert np.isnan(M.stored(x)[0, 32:]).all() and (M.stored(x)[0, :32] == 0).all()
