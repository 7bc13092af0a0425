"""Limits of attention, held on the host: no GPU needed."""
import ctypes as C

import pytest

from paper_2408_06995_amd import binding as B
from test_abi_adapt import attention_args


@pytest.mark.parametrize("scale,status", [(1e-40, -3), (1e-38, -3), (2.0 ** -101, -3), (2.0 ** 101, -3), (3e38, -3), (2.0 ** -100, 0), (2.0 ** 100, 0)])
def test_scales_whose_units_overflow_are_refused(scale, status):
    """(batch 0: a call that is accepted has nothing to launch)"""
    L, p = B.lib(), C.c_void_p(4096)
    a = attention_args(scale=scale, batch=0)
    assert L.fpq_attention(C.byref(a), p, p, p, p, p, None, 0, None) == status
    assert L.fpq_attention_backward(C.byref(a), *[p] * 9, None, 0, None) == status


@pytest.mark.parametrize("batch,kv_len", [(1, 1 << 30), (4, 1 << 29), (2, 1 << 30)])
def test_gradients_of_more_keys_than_a_launch_has_threads_are_refused(batch, kv_len):
    """2^24 blocks of keys, of 256 threads each (without a workspace, so that no call goes on to a launch)."""
    L, p = B.lib(), C.c_void_p(4096)
    a = attention_args(batch=batch, q_heads=2, kv_heads=2, q_len=1, kv_len=kv_len, head_dim=8)
    assert L.fpq_attention_backward(C.byref(a), *[p] * 9, None, 0, None) == -4
    assert L.fpq_attention(C.byref(a), p, p, p, p, p, None, 0, None) == -6
