"""Calls of attention over the cache with more work items than a launch has room for are refused, the ones below are not.

The workspace query makes the same checks as the call and needs no device.
"""

import ctypes

import pytest

import paper_2607_16190_amd as fva

A = 0x7F0000001000  # never dereferenced


def query(streams, H, KH, tokens, width, max_q, page=64):
    d = fva._Desc(1, H, tokens, 128, H * tokens * 128, 128, H * 128)
    n = ctypes.c_size_t(0)
    c = fva._Cache(20, KH, page, 128, A, A, A, A)
    st = fva.lib.fva_attn_cache_workspace_size(ctypes.byref(d), ctypes.byref(c), width, streams, max_q, ctypes.byref(n))
    if st == fva.FVA_ERR_UNSUPPORTED:
        call = fva.lib.fva_attn_cache(A, ctypes.byref(d), ctypes.byref(c), A, width, A, A, streams, max_q, 0, 0, ctypes.c_float(0), A, A,
                                      1 << 50, None)
        assert call == st
    return st


@pytest.mark.parametrize("streams,H,KH,tokens,width,max_q", [
    (1 << 20, 16, 16, 1 << 20, 100, 1),  # 17.8 million tiles of single tokens
    (1 << 24, 1, 1, 1 << 24, 4, 1),
    (1 << 24, 1, 1, 16, 100, 5000),  # streams without rows count, as lengths are not known here
    (1 << 20, 40, 40, 1 << 20, 4, 2000),
    (2**31 - 1, 1, 1, 2**31 - 1, 4, 1),
])
def test_too_many_work_items(streams, H, KH, tokens, width, max_q):
    assert query(streams, H, KH, tokens, width, max_q) == fva.FVA_ERR_UNSUPPORTED


@pytest.mark.parametrize("streams,H,KH,tokens,width,max_q", [
    (1 << 19, 16, 16, 1 << 19, 100, 1),
    (2048, 40, 40, 2048, 2000, 1),
    (2048, 40, 8, 2048 * 40, 2000, 60),
    (1, 40, 40, 1 << 23, 1 << 17, 1 << 23),  # 86 GB of Q: 2.6 million large tiles
    (1, 1, 1, 1 << 20, 1 << 23, 1),
])
def test_work_items_that_fit(streams, H, KH, tokens, width, max_q):
    assert query(streams, H, KH, tokens, width, max_q) == fva.FVA_OK
