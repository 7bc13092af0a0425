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


def adamw_tensor(**kw):
    t = B.fpq_adamw_tensor_t(param=4096, grad=8192, m=4096 * 3, v=4096 * 4, m_scale=4096 * 5, v_scale=4096 * 6, copy=None, n=1000, param_type=0, grad_type=1,
                             state_bits=8)
    for n, v in kw.items():
        setattr(t, n, v)
    return (B.fpq_adamw_tensor_t * 1)(t)


def test_adamw_refusals():
    L, p, out = B.lib(), C.c_void_p(4096), C.c_int64(0)
    plan = lambda a, n=1, at=p, size=1 << 20, o=C.byref(out): L.fpq_adamw_plan(a, n, at, size, o, None)
    for kw, status in ((dict(n=-1), -4), (dict(n=1 << 31), -4), (dict(param_type=2), -8), (dict(grad_type=-1), -8), (dict(state_bits=16), -8), (dict(reserved=1), -8),
                       (dict(param=None), -1), (dict(grad=None), -1), (dict(m=None), -1), (dict(v=None), -1), (dict(m_scale=None), -1), (dict(v_scale=None), -1),
                       (dict(param=4098), -5), (dict(grad=4097), -5), (dict(m=4098, state_bits=32), -5), (dict(v_scale=4098), -5), (dict(copy=4097), -5)):
        assert plan(adamw_tensor(**kw)) == status, kw
        assert L.fpq_adamw_plan_size(adamw_tensor(**kw), 1) == 0
    good = adamw_tensor()
    need = L.fpq_adamw_plan_size(good, 1)
    assert need == 16 + 80 and plan(good, size=need - 1) == -6 and plan(good, at=None) == -1 and plan(good, at=C.c_void_p(4104)) == -5
    assert plan(good, n=-1) == -4 and plan(None) == -1 and plan(good, o=None) == -1 and plan(None, n=0) == 0 and out.value == 0
    step = lambda pieces=1, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.0, t=1, at=p, gs=None: L.fpq_adamw_step(at, pieces, lr, b1, b2, eps, wd, t, gs, None)
    nan, inf = float("nan"), float("inf")
    for kw in (dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(b1=1.0), dict(b1=-0.1), dict(b1=nan), dict(b2=1.0), dict(b2=nan), dict(eps=0.0), dict(eps=nan),
               dict(eps=inf), dict(wd=-1.0), dict(wd=nan)):
        assert step(**kw) == -3, kw
    assert step(t=0) == -4 and step(pieces=-1) == -4 and step(at=None) == -1 and step(at=C.c_void_p(4104)) == -5 and step(gs=C.c_void_p(4098)) == -5
    assert step(pieces=0) == 0


def test_adamw_binding_checks():
    f, b = torch.zeros(300), torch.zeros(300, dtype=torch.uint8)
    s = torch.ones(2)
    B.adamw_tensors([(f, f, f, f, None, None, None), (f, f.bfloat16(), b, b, s, s, f.bfloat16())])
    for error, item in ((TypeError, (f.double(), f, f, f, None, None, None)), (TypeError, (f, f, f.double(), f.double(), None, None, None)),
                        (TypeError, (f, f, f, b, None, None, None)), (TypeError, (f, f, b, b, s, None, None)), (TypeError, (f, f, f, f, None, None, f)),
                        (ValueError, (f, f[:299], f, f, None, None, None)), (ValueError, (f, f, b, b, s, s[:1], None)),
                        (ValueError, (torch.zeros(600)[::2], f, f, f, None, None, None))):
        with pytest.raises(error):
            B.adamw_tensors([item])


def adapter_args(**kw):
    a = B.fpq_adapter_args_t(x_type=0, w_type=1, M=10, N=32, K=64, R=8, requests=2, adapters=3, scaling=4096, row_start=4096, adapter=4096, ld_x=64, ld_base=32, ld_y=32,
                             ld_grad_y=32, ld_grad_x_base=64, ld_grad_x=64)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def test_adapter_refusals():
    L, p, big = B.lib(), C.c_void_p(4096), 1 << 40
    fwd = lambda a, x=p, wa=p, wb=p, base=p, y=p, t=p, ws=p, n=big: L.fpq_adapter_apply(C.byref(a), x, wa, wb, base, y, t, ws, n, None)
    back = lambda a, ws=p, n=big, **kw: L.fpq_adapter_backward(C.byref(a), *[kw.get(v, p) for v in "x wa wb t gy gxb gx ga gb".split()], ws, n, None)
    assert L.fpq_adapter_apply(None, p, p, p, p, p, p, p, big, None) == -1
    for kw, status in ((dict(x_type=2), -8), (dict(w_type=-1), -8), (dict(x_type=1, w_type=0), -8), (dict(R=129), -8), (dict(R=0), -4), (dict(N=0), -4), (dict(K=0), -4),
                       (dict(M=-1), -4), (dict(adapters=0), -4), (dict(adapters=65536), -4), (dict(requests=-1), -4), (dict(K=1 << 28, R=8, ld_x=1 << 28), -4),
                       (dict(ld_x=63), -4), (dict(scaling=None), -1), (dict(row_start=None), -1), (dict(adapter=None), -1), (dict(scaling=4097), -5),
                       (dict(row_start=4098), -5), (dict(adapter=4098), -5)):
        assert fwd(adapter_args(**kw)) == status, kw
        assert back(adapter_args(**kw)) == status, kw
    for kw in (dict(ld_y=31), dict(ld_base=31)):
        assert fwd(adapter_args(**kw)) == -4
    for kw in (dict(ld_grad_y=31), dict(ld_grad_x=63), dict(ld_grad_x_base=63)):
        assert back(adapter_args(**kw)) == -4
    a = adapter_args()
    for name in ("x", "wa", "wb", "y"):
        assert fwd(a, **{name: None}) == -1 and fwd(a, **{name: C.c_void_p(4097)}) == -5
    assert fwd(a, base=C.c_void_p(4098)) == -5 and fwd(a, t=C.c_void_p(4098)) == -5
    for name in ("x", "wa", "wb", "t", "gy", "ga", "gb"):
        assert back(a, **{name: None}) == -1 and back(a, **{name: C.c_void_p(4097)}) == -5, name
    assert back(a, gx=C.c_void_p(4098)) == -5 and back(a, gxb=C.c_void_p(4098)) == -5
    assert L.fpq_adapter_workspace_size(10, 32, 64, 8, 2, 3) == 0              # the forward call needs none
    need = L.fpq_adapter_backward_workspace_size(10, 32, 64, 8, 2, 3)
    assert need > 0 and back(a, n=need - 1) == -6 and back(a, ws=None) == -6 and back(a, ws=C.c_void_p(4100)) == -5
    assert fwd(adapter_args(M=0)) == 0
    assert L.fpq_adapter_workspace_size(10, 32, 64, 129, 2, 3) == 0 and L.fpq_adapter_backward_workspace_size(10, 32, 0, 8, 2, 3) == 0


def test_adapter_binding_checks():
    x, a, b = torch.zeros(10, 64), torch.zeros(3, 8, 64), torch.zeros(3, 32, 8)
    s, start, of = torch.ones(3), torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    y, t = torch.zeros(10, 32), torch.zeros(10, 8)

    def refused(error, match, *args):
        with pytest.raises(error, match=match):
            B.fpq_adapter_apply(*args)

    refused(ValueError, "2 dimensions", x[0], a, b, s, start, of, y, y, t)
    refused(ValueError, "b \\[adapters", x, a, b[:2], s, start, of, y, y, t)
    refused(ValueError, "contiguous", x, torch.zeros(3, 16, 64)[:, :8], b, s, start, of, y, y, t)
    refused(ValueError, "contiguous", x, a, torch.zeros(3, 64, 8)[:, ::2], s, start, of, y, y, t)
    refused(ValueError, "the adapters' K", x[:, :32], a, b, s, start, of, y, y, t)
    refused(ValueError, "scaling", x, a, b, s[:2], start, of, y, y, t)
    refused(ValueError, "row_start", x, a, b, s, start[:2], of, y, y, t)
    refused(ValueError, "adapter", x, a, b, s, start, of.long(), y, y, t)
    refused(ValueError, "base", x, a, b, s, start, of, y[:5], y, t)
    refused(ValueError, "y:", x, a, b, s, start, of, None, y.bfloat16(), t)
    refused(ValueError, "t:", x, a, b, s, start, of, None, y, t[:5])
    refused(TypeError, "float32 or bfloat16", x.double(), a, b, s, start, of, None, y, t)
    refused(ValueError, "one type", x, a, b.bfloat16(), s, start, of, None, y, t)
    with pytest.raises(ValueError, match="grad_a"):
        B.fpq_adapter_backward(x, a, b, s, start, of, t, y, None, x, a[:2], b)


def test_adapter_ranks_above_16_that_are_packed():
    """Rows off the multiples of eight elements need a workspace in the forward call; others need aligned weights."""
    L = B.lib()
    assert L.fpq_adapter_workspace_size(10, 32, 64, 24, 2, 3) == 0 and L.fpq_adapter_workspace_size(10, 32, 63, 16, 2, 3) == 0
    need = L.fpq_adapter_workspace_size(10, 32, 64, 20, 2, 3)
    # three planes of bf16 for each adapter, both lengths in steps of 64 and the rank in steps of 32
    assert need >= 3 * 2 * 3 * 32 * (64 + 64) and L.fpq_adapter_workspace_size(10, 32, 63, 24, 2, 3) >= need
    p, off = C.c_void_p(4096), C.c_void_p(4104)

    def call(R, a, b, ws, n):
        return L.fpq_adapter_apply(C.byref(adapter_args(x_type=1, w_type=1, R=R)), p, a, b, p, p, None, ws, n, None)
    assert call(20, p, p, None, 0) == -6 and call(20, p, p, p, need - 1) == -6 and call(20, p, p, off, need) == -5
    assert call(24, off, p, None, 0) == -5 and call(24, p, off, None, 0) == -5
