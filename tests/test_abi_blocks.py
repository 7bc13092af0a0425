"""Refusals of the operators around the projections: documented codes before anything is launched, no GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2408_06995_amd import binding as B

P, ODD = C.c_void_p(4096), C.c_void_p(4097)                # never dereferenced: every call below fails validation first
E4M3, E2M1 = B.fmt((4, 3, 7, 448.0)), B.fmt((2, 1, 1, 6.0))
ROOM = 1 << 40


def with_(a, **kw):
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def test_block_refusals():
    L = B.lib()
    q = lambda x=P, t=0, M=4, K=40, ld=40, f=E4M3, mask=None, codes=P, scales=P: L.fpq_block_quantize(x, t, M, K, ld, f, mask, codes, scales, None)
    d = lambda codes=P, scales=P, M=4, K=40, f=E4M3, out=P, t=0, ld=40: L.fpq_block_dequantize(codes, scales, M, K, f, out, t, ld, None)
    for f, status in (((9, 3, 7, 0.0), -2), ((4, 3, 7, 0.0), -8), ((4, 3, 8, 0.0), -8), ((5, 2, 15, 57344.0), -8), ((2, 1, 2, 0.0), -8), ((2, 1, 1, 4.0), -8)):
        assert q(f=B.fmt(f)) == status and d(f=B.fmt(f)) == status, f
    assert q(t=2) == -8 and d(t=-1) == -8 and q(mask=P) == -8
    for kw in (dict(M=-1), dict(M=(1 << 28) + 1), dict(K=0), dict(K=(1 << 20) + 1), dict(ld=39), dict(ld=(1 << 20) + 1), dict(M=1 << 20, K=1 << 14, ld=1 << 14)):
        assert q(**kw) == -4 and d(**kw) == -4, kw
    for kw in (dict(codes=None), dict(scales=None)):
        assert q(**kw) == -1 and d(**kw) == -1
    assert q(x=None) == -1 and d(out=None) == -1 and q(x=ODD) == -5 and d(out=ODD) == -5 and q(codes=C.c_void_p(4104)) == -5 and d(codes=C.c_void_p(4104)) == -5
    assert q(M=0) == 0 and d(M=0) == 0 and q(M=0, x=None) == 0
    assert B.fpq_block_padded(1) == 32 and B.fpq_block_padded(64) == 64 and B.fpq_block_padded(0) == 0 and B.fpq_block_padded(-1) == 0


def linear(**kw):
    return with_(B.fpq_linear_args_t(type=1, M=20, N=48, K=40, ld_x=40, ld_y=48, ld_w=40, ld_grad_y=48, ld_grad_x=40, ld_grad_w=40), **kw)


SIZES = (dict(M=-1), dict(M=(1 << 28) + 1), dict(N=0), dict(K=0), dict(N=(1 << 20) + 1), dict(K=(1 << 20) + 1), dict(M=1 << 27, N=1 << 7, K=1))


def test_block_linear_refusals():
    L = B.lib()
    f = lambda a=None, x=P, codes=P, scales=P, bias=None, y=P, ws=P, n=ROOM: L.fpq_block_linear(C.byref(a or linear()), x, codes, scales, bias, y, ws, n, None)
    assert L.fpq_block_linear(None, P, P, P, None, P, P, ROOM, None) == -1
    for kw, status in ((dict(type=2), -8), (dict(reserved=1), -8), (dict(ld_x=39), -4), (dict(ld_y=47), -4), (dict(ld_y=1 << 21), -4), *((k, -4) for k in SIZES)):
        assert f(linear(**kw)) == status, kw
    for kw in ("x", "codes", "scales", "y"):
        assert f(**{kw: None}) == -1
    for kw in (dict(x=ODD), dict(y=ODD), dict(codes=C.c_void_p(4104)), dict(bias=C.c_void_p(4098))):
        assert f(**kw) == -5, kw
    need, many = L.fpq_block_linear_workspace_size(200, 48, 40, 1), linear(M=200)
    assert need > 0 and f(many, ws=None) == -6 and f(many, n=need - 1) == -6 and f(many, ws=C.c_void_p(4104)) == -5
    assert L.fpq_block_linear_workspace_size(64, 48, 40, 1) == 0
    assert f(linear(M=0), x=None, ws=None, n=0) == 0
    for bad in ((-1, 48, 40, 1), (20, 0, 40, 1), (20, 48, 40, 2), (20, 48, 1 << 21, 1)):
        assert L.fpq_block_linear_workspace_size(*bad) == 0 and L.fpq_linear_backward_workspace_size(*bad) == 0 and L.fpq_gated_workspace_size(*bad) == 0
        assert L.fpq_gated_backward_workspace_size(*bad) == 0


def test_linear_backward_refusals():
    L = B.lib()
    f = lambda a=None, x=P, xs=None, w=P, gy=P, gx=P, gw=P, gb=P, ws=P, n=ROOM: L.fpq_linear_backward(C.byref(a or linear()), x, xs, w, gy, gx, gw, gb, ws, n, None)
    assert L.fpq_linear_backward(None, P, None, P, P, P, P, P, P, ROOM, None) == -1
    for kw, status in ((dict(type=2), -8), (dict(reserved=1), -8), (dict(ld_x=39), -4), (dict(ld_w=39), -4), (dict(ld_grad_y=47), -4), (dict(ld_grad_x=39), -4),
                       (dict(ld_grad_w=39), -4), *((k, -4) for k in SIZES)):
        assert f(linear(**kw)) == status, kw
    assert f(gy=None) == -1 and f(x=None) == -1 and f(w=None) == -1
    for kw in (dict(x=ODD), dict(x=C.c_void_p(4104), xs=P), dict(w=ODD), dict(gy=ODD), dict(gx=ODD), dict(gw=ODD), dict(gb=C.c_void_p(4098))):
        assert f(**kw) == -5, kw
    need = L.fpq_linear_backward_workspace_size(20, 48, 40, 1)
    assert need > 0 and f(ws=None) == -6 and f(n=need - 1) == -6 and f(ws=C.c_void_p(4104)) == -5
    assert f(gx=None, gw=None, gb=None) == 0


def gated(**kw):
    return with_(B.fpq_gated_args_t(type=1, act=0, M=20, N=48, K=40, ld_x=40, ld_w=40, ld_h=48, ld_grad_h=48, ld_grad_x=40, ld_grad_w=40), **kw)


def test_gated_refusals():
    L = B.lib()
    f = lambda a=None, x=P, w=P, bias=None, h=P, pre=None, ps=None, ws=P, n=ROOM: L.fpq_gated(C.byref(a or gated()), x, w, bias, h, pre, ps, ws, n, None)
    b = lambda a=None, x=P, xs=None, w=P, pre=P, ps=None, gh=P, gx=P, gw=P, gb=P, ws=P, n=ROOM: L.fpq_gated_backward(
        C.byref(a or gated()), x, xs, w, pre, ps, gh, gx, gw, gb, ws, n, None)
    assert L.fpq_gated(None, P, P, None, P, None, None, P, ROOM, None) == -1 and L.fpq_gated_backward(None, P, None, P, P, None, P, P, P, P, P, ROOM, None) == -1
    sizes = [dict(k) for k in SIZES] + [dict(N=(1 << 19) + 1), dict(N=-5), dict(N=1 << 62)]
    for kw, status in ((dict(type=2), -8), (dict(act=2), -8), (dict(act=-1), -8), (dict(ld_w=39), -4), *((k, -4) for k in sizes)):
        assert f(gated(**kw)) == status and b(gated(**kw)) == status, kw
    assert f(gated(ld_x=39)) == -4 and f(gated(ld_h=47)) == -4 and b(gated(ld_x=39)) == -4 and b(gated(ld_grad_h=47)) == -4
    assert b(gated(ld_grad_x=39)) == -4 and b(gated(ld_grad_w=39)) == -4
    for kw in ("x", "w", "h"):
        assert f(**{kw: None}) == -1 and f(**{kw: ODD}) == -5
    assert f(ps=P) == -1 and f(pre=ODD) == -5 and f(pre=C.c_void_p(4104), ps=P) == -5 and f(bias=C.c_void_p(4098)) == -5
    for kw in ("x", "w", "pre", "gh"):
        assert b(**{kw: None}) == -1 and b(**{kw: ODD}) == -5
    for kw in (dict(x=C.c_void_p(4104), xs=P), dict(pre=C.c_void_p(4104), ps=P), dict(gx=ODD), dict(gw=ODD), dict(gb=C.c_void_p(4098))):
        assert b(**kw) == -5, kw
    for call, size in ((f, L.fpq_gated_workspace_size), (b, L.fpq_gated_backward_workspace_size)):
        a = gated(type=0, ld_x=40)
        need = size(20, 48, 40, 0)
        assert need > 0 and call(a, ws=None) == -6 and call(a, n=need - 1) == -6 and call(a, ws=C.c_void_p(4104)) == -5
    assert f(gated(M=0), x=None, ws=None, n=0) == 0 and b(gx=None, gw=None, gb=None) == 0


def norm(**kw):
    return with_(B.fpq_norm_args_t(type=1, eps=1e-6, M=20, K=40, ld_x=40, ld_residual=40, ld_sum=40, ld_y=40, ld_grad_y=40, ld_grad_sum=40, ld_grad_x=40), **kw)


def test_norm_refusals():
    L = B.lib()
    f = lambda a=None, x=P, res=P, w=P, sum=P, y=P, rstd=P, codes=P, fm=E4M3, scale=1.0, dev=None, cs=None: L.fpq_rms_norm(
        C.byref(a or norm()), x, res, w, sum, y, rstd, codes, fm, scale, dev, cs, None)
    b = lambda a=None, sum=P, w=P, rstd=P, gy=P, gs=P, gx=P, gw=P, ws=P, n=ROOM: L.fpq_rms_norm_backward(C.byref(a or norm()), sum, w, rstd, gy, gs, gx, gw, ws, n, None)
    assert L.fpq_rms_norm(None, P, P, P, P, P, P, None, E4M3, 1.0, None, None, None) == -1 and L.fpq_rms_norm_backward(None, P, P, P, P, P, P, P, P, ROOM, None) == -1
    for kw, status in ((dict(type=2), -8), (dict(M=-1), -4), (dict(K=0), -4), (dict(K=(1 << 20) + 1), -4), (dict(M=1 << 27, K=1 << 8), -4), (dict(ld_sum=39), -4)):
        assert f(norm(**kw)) == status and b(norm(**kw)) == status, kw
    for kw in (dict(ld_x=39), dict(ld_residual=39), dict(ld_y=1 << 21)):
        assert f(norm(**kw)) == -4
    for kw in (dict(ld_grad_y=39), dict(ld_grad_sum=39), dict(ld_grad_x=39)):
        assert b(norm(**kw)) == -4
    for eps in (-1.0, float("nan"), float("inf")):
        assert f(norm(eps=eps)) == -3
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert f(scale=scale) == -3
    assert f(fm=B.fmt((9, 3, 7, 0.0))) == -2
    assert f(x=None) == -1 and f(sum=None) == -1 and f(codes=None, cs=P) == -1
    for kw in ("x", "res", "sum", "y"):
        assert f(**{kw: ODD}) == -5
    for kw in ("w", "rstd"):
        assert f(**{kw: C.c_void_p(4098)}) == -5
    assert f(codes=C.c_void_p(4104)) == -5 and f(dev=C.c_void_p(4098)) == -5
    for kw in ("sum", "rstd", "gy"):
        assert b(**{kw: None}) == -1
    for kw in ("sum", "gy", "gs", "gx"):
        assert b(**{kw: ODD}) == -5
    for kw in ("w", "rstd", "gw"):
        assert b(**{kw: C.c_void_p(4098)}) == -5
    need = L.fpq_rms_norm_backward_workspace_size(20, 40)
    assert need > 0 and b(ws=None) == -6 and b(n=need - 1) == -6 and b(ws=C.c_void_p(4104)) == -5 and L.fpq_rms_norm_backward_workspace_size(20, 0) == 0
    assert f(norm(M=0), x=None) == 0 and b(gx=None, gw=None) == 0


def test_binding_checks():
    x, w, u8 = torch.zeros(6, 40), torch.zeros(12, 40), lambda *s: torch.zeros(s, dtype=torch.uint8)

    def refused(error, match, call, *args):
        with pytest.raises(error, match=match):
            call(*args)

    q = B.fpq_block_quantize
    refused(ValueError, "2 dimensions", q, x[0], (4, 3, 7, 448.0), None, u8(6, 64), u8(6, 2))
    refused(ValueError, "codes", q, x, (4, 3, 7, 448.0), None, u8(6, 40), u8(6, 2))
    refused(ValueError, "codes", q, x, (2, 1, 1, 6.0), None, u8(6, 64), u8(6, 2))
    refused(ValueError, "scales", q, x, (4, 3, 7, 448.0), None, u8(6, 64), u8(6, 1))
    refused(ValueError, "not contiguous", q, x, (4, 3, 7, 448.0), None, u8(64, 6).t(), u8(6, 2))
    refused(ValueError, "mask", q, x, (2, 1, 1, 6.0), u8(6, 39), u8(6, 32), u8(6, 2))
    refused(TypeError, "float32 or bfloat16", q, x.half(), (4, 3, 7, 448.0), None, u8(6, 64), u8(6, 2))
    refused(ValueError, "neighbours", q, torch.zeros(40, 6).t(), (4, 3, 7, 448.0), None, u8(6, 64), u8(6, 2))
    d = B.fpq_block_dequantize
    refused(ValueError, "scales", d, u8(6, 64), u8(6, 1), (4, 3, 7, 448.0), x)
    lin = B.fpq_block_linear
    refused(ValueError, "codes", lin, x, u8(12, 64), u8(12, 2), None, torch.zeros(6, 12))
    refused(ValueError, "bias", lin, x, u8(12, 32), u8(12, 2), torch.zeros(11), torch.zeros(6, 12))
    refused(ValueError, "y: 6 rows", lin, x, u8(12, 32), u8(12, 2), None, torch.zeros(5, 12))
    refused(ValueError, "y: 6 rows", lin, x, u8(12, 32), u8(12, 2), None, torch.zeros(6, 12).bfloat16())
    bw, gy = B.fpq_linear_backward, torch.zeros(6, 12)
    refused(ValueError, "w: 12 rows", bw, x, None, w[:11], gy, x, w, None)
    refused(ValueError, "x: 6 rows", bw, x[:5], None, w, gy, x, w, None)
    refused(ValueError, "x: codes", bw, u8(6, 40), u8(6, 2), w, gy, x, w, None)
    refused(ValueError, "x_scales", bw, u8(6, 64), u8(6, 3), w, gy, x, w, None)
    refused(ValueError, "grad_x", bw, x, None, w, gy, x[:, :39], w, None)
    refused(ValueError, "grad_w", bw, x, None, w, gy, x, w[:5], None)
    refused(ValueError, "grad_bias", bw, x, None, w, gy, x, w, torch.zeros(13))
    refused(TypeError, "a tensor", bw, x, None, None, gy, x, w, None)
    ga, h = B.fpq_gated, torch.zeros(6, 6)
    refused(ValueError, "w: 12 rows", ga, x, w[:10], None, 0, h)
    refused(ValueError, "bias", ga, x, w, torch.zeros(6), 0, h)
    refused(ValueError, "pre: 6 rows", ga, x, w, None, 0, h, torch.zeros(6, 6))
    refused(ValueError, "pre: not contiguous", ga, x, w, None, 0, h, torch.zeros(6, 13)[:, :12])
    refused(ValueError, "pre: codes", ga, x, w, None, 0, h, u8(6, 12), u8(6, 2))
    gb = B.fpq_gated_backward
    refused(TypeError, "pre", gb, x, None, w, None, None, 0, h, x, w, None)
    refused(ValueError, "grad_bias", gb, x, None, w, torch.zeros(6, 12), None, 0, h, x, w, torch.zeros(6))
    n = B.fpq_rms_norm
    refused(ValueError, "residual", n, x, x[:5], None, 1e-6, x, x)
    refused(ValueError, "w: 40", n, x, x, torch.zeros(39), 1e-6, x, x)
    refused(ValueError, "codes", n, x, x, None, 1e-6, x, x, None, u8(6, 40), (4, 3, 7, 448.0), 1.0)
    refused(ValueError, "codes", n, x, x, None, 1e-6, x, x, None, u8(6, 48), None, None, None, u8(6, 2))
    refused(ValueError, "rstd", n, x, x, None, 1e-6, x, x, torch.zeros(5))
    refused(ValueError, "grad_w", B.fpq_rms_norm_backward, x, None, torch.zeros(6), x, None, x, torch.zeros(6))
