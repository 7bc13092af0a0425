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
