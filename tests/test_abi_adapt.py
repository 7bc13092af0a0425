"""Refusals of the operators for adapting a model: documented codes before anything is launched, no GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2408_06995_amd import binding as B


def attention_args(**kw):
    a = B.fpq_attention_args_t(type=0, batch=2, q_heads=4, kv_heads=2, q_len=8, kv_len=9, head_dim=16, scale=0.25)
    for n in ("q", "o", "grad_o", "grad_q"):
        getattr(a, n + "_strides")[:] = [8 * 4 * 16, 4 * 16, 16]
    for n in ("k", "v", "grad_k", "grad_v"):
        getattr(a, n + "_strides")[:] = [9 * 2 * 16, 2 * 16, 16]
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def test_attention_refusals():
    L, p = B.lib(), C.c_void_p(4096)                       # never dereferenced: every call below fails validation first
    fwd = lambda a, q=p, k=p, v=p, o=p, lse=p, ws=None, n=0: L.fpq_attention(C.byref(a), q, k, v, o, lse, ws, n, None)
    assert L.fpq_attention(None, p, p, p, p, p, None, 0, None) == -1
    for kw, status in ((dict(type=2), -8), (dict(causal=2), -8), (dict(head_dim=161), -8), (dict(head_dim=0), -4), (dict(q_heads=3), -4), (dict(kv_heads=0), -4),
                       (dict(batch=-1), -4), (dict(kv_len=(1 << 30) + 1), -4), (dict(q_len=1 << 30, q_heads=8), -4), (dict(scale=0.0), -3),
                       (dict(scale=float("nan")), -3), (dict(scale=float("inf")), -3), (dict(scale=-1.0), -3),
                       (dict(batch=1 << 20, q_len=4096), -4)):
        assert fwd(attention_args(**kw)) == status, kw
        assert L.fpq_attention_backward(C.byref(attention_args(**kw)), p, p, p, p, p, p, p, p, p, None, 0, None) == status, kw
        assert L.fpq_attention_workspace_size(C.byref(attention_args(**kw))) == 0
    a = attention_args()
    for name in ("q", "k", "v", "o"):
        assert fwd(a, **{name: None}) == -1
        assert fwd(a, **{name: C.c_void_p(4098)}) == -5
    assert fwd(a, lse=C.c_void_p(4098)) == -5 and fwd(attention_args(kv_lens=4098)) == -5
    assert fwd(attention_args(batch=0)) == 0 and fwd(attention_args(q_len=0)) == 0
    long = attention_args(q_len=1, kv_len=8192)
    need = L.fpq_attention_workspace_size(C.byref(long))
    assert need > 0 and fwd(long) == -6 and fwd(long, ws=p, n=need - 1) == -6 and fwd(long, ws=C.c_void_p(4100), n=need) == -5
    back = lambda a, ws=p, n=1 << 30, **kw: L.fpq_attention_backward(C.byref(a), *[kw.get(x, p) for x in "q k v o lse go gq gk gv".split()], ws, n, None)
    for name in "q k v o lse go gq gk gv".split():
        assert back(a, **{name: None}) == -1, name
        assert back(a, **{name: C.c_void_p(4098)}) == -5, name
    need = L.fpq_attention_backward_workspace_size(C.byref(a))
    assert need >= 4 * 2 * 4 * 8 and back(a, n=need - 1) == -6 and back(a, ws=None) == -6 and back(a, ws=C.c_void_p(4100)) == -5
    assert back(attention_args(batch=0)) == 0 and back(attention_args(q_len=0, kv_len=0)) == 0


def test_attention_binding_checks():
    q, k = torch.zeros(2, 8, 4, 16), torch.zeros(2, 9, 2, 16)
    lse = torch.zeros(2, 4, 8)

    def refused(error, match, *args):
        with pytest.raises(error, match=match):
            B.fpq_attention(*args)

    refused(ValueError, "4 dimensions", q[0], k, k, q, lse, 1.0)
    refused(ValueError, "neighbours", q.transpose(2, 3), k, k, q, lse, 1.0)
    refused(ValueError, "shape of k", q, k, k[:, :5], q, lse, 1.0)
    refused(ValueError, "shape of q", q, k, k, q[:, :5], lse, 1.0)
    refused(ValueError, "samples and the head", q, k[:1], k[:1], q, lse, 1.0)
    refused(ValueError, "lse", q, k, k, q, lse[:, :2], 1.0)
    refused(ValueError, "kv_lens", q, k, k, q, lse, 1.0, 0, torch.zeros(3, dtype=torch.int32))
    refused(ValueError, "kv_lens", q, k, k, q, lse, 1.0, 0, torch.zeros(2, dtype=torch.int64))
    refused(TypeError, "float32 or bfloat16", q.half(), k, k, q, lse, 1.0)
    refused(ValueError, "one type", q, k.bfloat16(), k, q, lse, 1.0)
    with pytest.raises(ValueError, match="gradients"):
        B.fpq_attention_backward(q, k, k, q, lse, q, q, k[:, :3], k, 1.0)
    with pytest.raises(ValueError, match="gradients"):
        B.fpq_attention_backward(q, k, k, q, lse, q.bfloat16(), q, k, k, 1.0)
