"""Limits of the calls on a paged whole-token cache that are found on the host.  Addresses here are made up and never dereferenced."""
import ctypes as C

import pytest

import paper_2506_18226_b200 as A
from paper_2506_18226_b200 import binding as B

P = 0x10000000      # a 256-byte aligned address


def _rotary(head_dim, pairs, halves):
    r = B.AdsaRotary()
    assert A.load().adsa_rotary_init(C.byref(r), head_dim, 1, (C.c_int32 * 1)(pairs), halves, 1, 0.0) == 0
    return r


@pytest.mark.parametrize("halves", [0, 1])
@pytest.mark.parametrize("heads", [2**23, 2**25, 2**26, 2**27 + 5, 2**31 - 1])
def test_more_heads_than_a_grid_holds_are_refused(heads, halves):
    """Their units (up to one an element) pass 32 bits."""
    r = _rotary(64, 32, halves)
    assert A.load().adsa_rope_axes(C.byref(r), 0, P + 2, 64, 64, P, 1, heads, P + 2, 64, 64, None) == B.EINVAL
    kv = B.AdsaPagedKv(P, P, 0, 10, 2, 16, 64, 64)
    assert A.load().adsa_paged_append(C.byref(kv), P, 1, 3, P, None, 1, P + 2, 128, 64, P, 128, 64, C.byref(r), P, P, heads, 0, 64, P, 0, 64,
                                      None, None) == B.EINVAL
