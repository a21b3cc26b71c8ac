"""Store copies of no tokens: nothing is looked at, nothing launched, nothing refused but what is wrong without tokens too (no GPU
needed)."""
import ctypes

import pytest

import paper_2512_00504_b200 as gkv

A = 1 << 20     # an aligned address that is never looked at


@pytest.mark.parametrize("strides", [(0, 0, 0), (4096, 256, 0), (0, 256, 128), (1 << 62, 1 << 62, 1 << 62)])
@pytest.mark.parametrize("k,v", [(None, None), (A, A)])
def test_no_tokens_do_nothing_whatever_the_strides(strides, k, v):
    gkv.build_library()
    s = gkv.gkv_store(format=gkv.GKV_STORE_INT8, batch=6, n_q_heads=8, n_kv_heads=2, head_dim=128, capacity=100, k=A, v=A, k_scale=A, v_scale=A)
    for f in (gkv.lib().gkv_store_write, gkv.lib().gkv_store_read):
        assert f(ctypes.byref(s), k, v, *strides, None, None, 0, None) == gkv.GKV_OK
        assert f(ctypes.byref(s), k, v, 4096, 256, 4, None, None, 0, None) == gkv.GKV_ERR_INVALID_ARG
