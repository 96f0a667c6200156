"""Refusals of the growing-chunk, shared-link and block-index calls that need no store: on the host."""
import ctypes

import pytest

from paper_2602_01519_amd import pic


@pytest.mark.parametrize("call", [
    lambda L: L.pic_store_open(None, 1, 5), lambda L: L.pic_store_append(None, None, None),
    lambda L: L.pic_store_truncate(None, 0, None, None, None),
    lambda L: L.pic_link_shared(None, None, None, 1, None, None, None, 1.0, None, None, None),
    lambda L: L.pic_link_shared(None, ctypes.byref(pic.LinkReq()), ctypes.byref(pic.LinkGroups()), 1, None, None, None,
                                1.0, None, None, None),
    lambda L: L.pic_link_shared_plan_create(None, None, None, 1, None),
    lambda L: L.pic_index_create(None, None), lambda L: L.pic_index_update(None, 0, 0, None, None),
    lambda L: L.pic_link_sparse(None, None, 1, 1, 0, 0, None, None, None, 1.0, None, None, None, None)])
def test_null_handles(call):
    assert call(pic.lib()) == pic.ERR_INVALID and pic.last_error()


def test_results_are_cleared():
    for create in (lambda out: pic.lib().pic_index_create(None, out),
                   lambda out: pic.lib().pic_link_shared_plan_create(None, None, None, 1, out)):
        h = ctypes.c_void_p(1)
        assert create(ctypes.byref(h)) == pic.ERR_INVALID and not h.value
    assert pic.lib().pic_index_destroy(None) == pic.OK
