"""Tensors of more than 2^31 elements in the operators around the projections: the last rows are what a call for them alone gives.  Whole
numbers, whose products and sums are exact in any order."""
import pytest
import torch

from paper_2408_06995_amd import binding as B
from gpu_util import DEV
from test_gpu_blocks import E2M1, E4M3, TYPES, room

pytestmark = pytest.mark.gpu

TAIL = 300


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def ints(seed, top, *shape):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-top, top + 1, shape, generator=g, device=DEV, dtype=torch.int8)


def raw(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_norm(t):
    print(t, flush=True)
    M, K = (1 << 25) + 77, 72
    x, res = (ints(i, 3, M, K).to(TYPES[t]) for i in range(2))
    assert x.numel() > 1 << 31
    total, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(M, device=DEV)
    codes, scales = raw(M * 96).view(M, 96), raw(M * 3).view(M, 3)
    B.fpq_rms_norm(x, res, None, 1e-3, total, y, rstd, codes, None, None, None, scales)
    s = [torch.empty_like(v[:TAIL]) for v in (total, y, rstd, codes, scales)]
    B.fpq_rms_norm(x[-TAIL:], res[-TAIL:], None, 1e-3, s[0], s[1], s[2], s[3], None, None, None, s[4])
    # (fewer rows take other threads, whose sums of whole numbers are the same)
    for a, b in zip((total, y, rstd, codes, scales), s):
        assert torch.equal(a[-TAIL:], b)
    gy = ints(5, 2, M, K).to(TYPES[t])
    gx, gw = torch.empty_like(x), torch.empty(K, device=DEV)
    ones = torch.ones(M, device=DEV)
    B.fpq_rms_norm_backward(total, None, ones, gy, None, gx, gw, room(B.fpq_rms_norm_backward_workspace_size(M, K)))
    # partial sums of whole numbers below 2^24 in each workgroup and in all: exact
    want = sum((a.double() * b.double()).sum(0) for a, b in zip(total.split(1 << 22), gy.split(1 << 22)))
    assert want.abs().max() < 1 << 24 and torch.equal(gw.double(), want)
    sx = torch.empty(TAIL, K, dtype=TYPES[t], device=DEV)
    B.fpq_rms_norm_backward(total[-TAIL:], None, ones[-TAIL:], gy[-TAIL:], None, sx, None)
    assert torch.equal(gx[-TAIL:], sx)


@pytest.mark.parametrize("f", [E4M3, E2M1], ids=["e4m3", "e2m1"])
def test_blocks(f):
    M, K = (1 << 25) + 77, 72
    per = 96 if f is E4M3 else 48
    x = ints(1, 100, M, K).to(torch.bfloat16)
    codes, scales = raw(M * per).view(M, per), raw(M * 3).view(M, 3)
    B.fpq_block_quantize(x, f, None, codes, scales)
    c, s = raw(TAIL * per).view(TAIL, per), raw(TAIL * 3).view(TAIL, 3)
    B.fpq_block_quantize(x[-TAIL:], f, None, c, s)
    assert torch.equal(codes[-TAIL:], c) and torch.equal(scales[-TAIL:], s)
    out, o = torch.empty_like(x), torch.empty(TAIL, K, dtype=torch.bfloat16, device=DEV)
    B.fpq_block_dequantize(codes, scales, f, out)
    B.fpq_block_dequantize(c, s, f, o)
    assert torch.equal(out[-TAIL:], o)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_linear_gradients(t):
    print(t, flush=True)
    M, N, K = (1 << 25) + 77, 72, 40
    # whole numbers up to 3 are themselves as blocks, whose scale is 2^-7 or 2^-8
    x, gy, w = ints(1, 3, M, K).to(TYPES[t]), ints(2, 2, M, N).to(TYPES[t]), ints(3, 2, N, K).to(TYPES[t])
    codes, scales = raw(M * 64).view(M, 64), raw(M * 2).view(M, 2)
    B.fpq_block_quantize(x, E4M3, None, codes, scales)
    gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device=DEV)
    B.fpq_linear_backward(codes, scales, w, gy, gx, gw, gb, room(B.fpq_linear_backward_workspace_size(M, N, K, int(t == "bf16"))))
    at = slice(M - TAIL, M)
    assert torch.equal(gx[at].double(), (gy[at].double() @ w.double()))
    want_w = sum(a.double().t() @ b.double() for a, b in zip(gy.split(1 << 22), x.split(1 << 22)))
    want_b = sum(a.double().sum(0) for a in gy.split(1 << 22))
    assert want_w.abs().max() < 1 << 24 and torch.equal(gw, want_w.to(TYPES[t])) and torch.equal(gb.double(), want_b)


def test_gated():
    M, N, K = (1 << 24) + 77, 136, 16
    t = torch.bfloat16
    x, w = ints(1, 2, M, K).to(t), (ints(2, 2, 2 * N, K).to(t) * 0.25)
    gh = ints(3, 2, M, N).to(t)
    Np = 160

    def call(x, gh, M):
        h, pre, scales = torch.empty(M, N, dtype=t, device=DEV), raw(M * 2 * Np).view(M, -1), raw(M * 2 * Np // 32).view(M, -1)
        B.fpq_gated(x, w, None, B.FPQ_GATE_SILU, h, pre, scales, room(B.fpq_gated_workspace_size(M, N, K, 1)))
        gx = torch.empty(M, K, dtype=t, device=DEV)
        B.fpq_gated_backward(None, None, w, pre, scales, B.FPQ_GATE_SILU, gh, gx, None, None, room(B.fpq_gated_backward_workspace_size(M, N, K, 1)))
        return h, pre, scales, gx

    many, few = call(x, gh, M), call(x[-TAIL:], gh[-TAIL:], TAIL)
    assert many[1].numel() > 1 << 31
    for a, b in zip(many[:3], few[:3]):
        assert torch.equal(a[-TAIL:], b)
    # (sums of 272 rounded products in another order: two roundings apart, and what the sum of fp32 magnitudes allows)
    a, b = many[3][-TAIL:].double(), few[3].double()
    assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + 2 * 272 * 2.0 ** -24 * 272 * 64).all()


def test_layer_on_4_bit_blocks():
    M, N, K = (1 << 25) + 77, 72, 40
    x, w = ints(1, 3, M, K).to(torch.bfloat16), ints(2, 3, N, K).float()
    codes, scales = raw(N * 32).view(N, 32), raw(N * 2).view(N, 2)
    B.fpq_block_quantize(w, E2M1, None, codes, scales)                   # (whole numbers up to 3 are themselves)
    y = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    B.fpq_block_linear(x, codes, scales, None, y, room(B.fpq_block_linear_workspace_size(M, N, K, 1)))
    assert y.numel() > 1 << 31 and torch.equal(y[-TAIL:], (x[-TAIL:].float() @ w.t()).bfloat16())
