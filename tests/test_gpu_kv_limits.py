"""Sizes that dcl_kv_attention refuses: decided on the host, no pointer is followed."""
import ctypes

import pytest

import paper_2607_20467_gb300 as dcl

pytestmark = pytest.mark.gpu

P = 0x7000_0000  # never dereferenced: each call is refused


@pytest.mark.parametrize("page_len", [16, 64, 256])
def test_positions_that_a_table_may_address(page_len):
    """The kernels look past a sequence's end in 32 bits, so that a table stops short of 2^31 positions."""
    import __graft_entry__
    __graft_entry__.build()
    L = dcl.lib()
    cache = dcl.KvCacheDesc(n_pages=4, page_len=page_len, n_kv_heads=2, head_dim=64, format=1, k_dev=P, v_dev=P,
                            k_exp_dev=P, v_exp_dev=P)
    most = (2 ** 31 - 4096) // page_len
    with dcl.Context(None, 1, 1) as ctx:
        for pages in (most + 1, (2 ** 31 - 1) // page_len, 2 ** 31 // page_len, 2 ** 31 - 1):
            st = L.dcl_kv_attention(ctx.ptr, ctypes.byref(cache), P, 256, P, P, pages, P, 1, 1, 1, 4, 0, 0.0, P, None)
            assert st == dcl.DCL_ERR_INVALID_ARG
            assert b"2^31 - 4096" in L.dcl_last_error(ctx.ptr)
