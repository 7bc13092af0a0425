"""Products of the operators around the projections in the tiles that no other test runs: layers on 4-bit blocks in large tiles and in slices, gated
projections of 17 to 64 rows on weights that the L2 does not hold, gradients of few rows, norms of odd widths and large ones in place.  Of large results rows at the ends and at
random, in full length."""
import numpy as np
import pytest
import torch

import test_gpu_blocks
import test_gpu_norm
from oracle import blocks
from paper_2408_06995_amd import binding as B
from gpu_util import DEV
from test_gpu_blocks import E2M1, TYPES, host, nan, quantize, rows, within
from test_gpu_blocks_edges import guarded  # noqa: F401
from test_gpu_gated import Call

pytestmark = pytest.mark.gpu


def some(n, seed, count=40):
    return np.unique(np.concatenate([[0, 1, n - 2, n - 1], np.random.RandomState(seed).randint(0, n, count)]))


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1000, 3000, 520), (1030, 1290, 5120), (700, 5121, 500),      # 128 x 128 with four stages, one slice and two
                                   (2000, 2600, 300), (2049, 2049, 100), (2048, 1280, 5120),      # 128 x 128
                                   (2051, 5001, 264), (3001, 3001, 200), (3300, 2600, 104),       # 192 x 256
                                   (3839, 4350, 136), (3839, 4350, 600),                          # 256 x 256
                                   (300, 520, 4000), (130, 131, 5000), (777, 1300, 2000)])        # 64 x 64, slices
def test_layers_on_4_bit_blocks(M, N, K, t, guarded):  # noqa: F811
    print(M, N, K, t, flush=True)
    g = torch.Generator().manual_seed(M + N)
    x, w, bias = rows(g, M, K, TYPES[t]), rows(g, N, K, torch.float32), torch.randn(N, generator=g).to(DEV)
    codes, scales = quantize(w, E2M1)
    wv = blocks.block_values(blocks.unpack(codes.cpu().numpy()), scales.cpu().numpy(), 4, K)
    ws, ms = guarded(B.fpq_block_linear_workspace_size(M, N, K, int(t == "bf16"))), some(M, N)
    for b in (bias, None):
        y = nan(M, N + 3, t=TYPES[t])
        B.fpq_block_linear(x, codes, scales, b, y[:, :N], ws)
        within("y", y[ms, :N], *blocks.block_linear(host(x[ms]), wv, None if b is None else host(b), t == "bf16"))
        assert y[:, :N].isfinite().all() and y[:, N:].isnan().all()


@pytest.mark.parametrize("keep", ["type", "blocks", None])
@pytest.mark.parametrize("M,N,K", [(17, 4200, 2048), (32, 2101, 4097), (25, 4801, 1800), (40, 4200, 2048), (64, 2101, 4097)])
def test_gated_tokens_on_large_weights(M, N, K, keep, guarded):  # noqa: F811
    print(M, N, K, keep, flush=True)
    c = Call(M, N, K, "bf16", "silu" if M % 2 else "gelu", bias=M != 25)
    h, pre, scales = c.forward(keep)
    want, off, ag, d_ag = blocks.gated(host(c.x), host(c.w), None if c.bias is None else host(c.bias), c.act, True)
    within("h", h, want, off)
    if keep:
        c.check_kept(pre, scales, ag, d_ag)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(3, 1000, 300), (17, 2000, 520), (32, 1283, 333), (20, 6000, 1000)])
def test_gradients_of_few_rows(M, N, K, t, guarded):  # noqa: F811
    """The gradient of x alone and beside the others, of linear layers and of gated projections."""
    print(M, N, K, t, flush=True)
    x, scales, w, gy = test_gpu_blocks.linear_case(M, N, K, t, True)
    xv, bf16 = blocks.block_values(x.cpu().numpy(), scales.cpu().numpy(), 8, K), int(t == "bf16")
    want = blocks.linear_backward(xv, host(w), host(gy), t == "bf16")
    for which in ((True, False, False), (True, True, True), (True, True, False)):
        out = [nan(*s, t=d) if on else None for on, s, d in zip(which, ((M, K), (N, K), (N,)), (TYPES[t], TYPES[t], torch.float32))]
        B.fpq_linear_backward(x, scales, w, gy, *out, guarded(B.fpq_linear_backward_workspace_size(M, N, K, bf16)))
        for name, got, ref in zip(("grad_x", "grad_w", "grad_bias"), out, want):
            if got is not None:
                within(name, got, *ref)
    c = Call(M, N // 2, K, t)
    pre, s, gx, _, _ = c.check("type")
    within("grad_x alone", c.backward(pre, s, gw=False, gb=False)[0], *blocks.gated_backward(host(c.x), host(c.w), *c.kept_values(pre, s), c.act, host(c.gh), t == "bf16")[0])


def test_gradient_of_x_in_tiles_of_256(guarded):  # noqa: F811
    M, N, K = 3839, 600, 4350
    x, _, w, gy = test_gpu_blocks.linear_case(M, N, K, "bf16", False)
    gx, ms = nan(M, K, t=torch.bfloat16), some(M, N)
    B.fpq_linear_backward(None, None, w, gy, gx, None, None, guarded(B.fpq_linear_backward_workspace_size(M, N, K, 1)))
    within("grad_x", gx[ms], *blocks.product(host(gy[ms]), host(w).T, blocks.rounding(True)))
    assert gx.isfinite().all()


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(7, 4097, 200), (16, 5001, 333), (16, 16383, 96)])
def test_few_rows_of_many_columns(M, N, K, t):
    test_gpu_blocks.test_layers_on_4_bit_blocks(M, N, K, 3, t)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K", [(3, 777), (700, 1001), (5, 2047), (40, 3001), (2, 4095)])
def test_norm_of_odd_widths(M, K, t):
    print(M, K, t, flush=True)
    test_gpu_norm.check(M, K, t)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K", [(3000, 12000), (3001, 11999), (6000, 5120), (40000, 320)])
def test_large_norms_in_place(M, K, t):
    """Results that the L2 does not hold, over what they came from: rows in registers and rows read twice."""
    print(M, K, t, flush=True)
    g = torch.Generator(device=DEV).manual_seed(K)
    x, res, gy, gs = (torch.randn(M, K, generator=g, device=DEV).to(TYPES[t]) for _ in range(4))
    w = 1 + 0.3 * torch.randn(K, generator=g, device=DEV)
    total, y, rstd = nan(M, K, t=TYPES[t]), nan(M, K, t=TYPES[t]), nan(M)
    B.fpq_rms_norm(x, res, w, 1e-6, total, y, rstd)
    assert torch.equal(total, (x.float() + res.float()).to(TYPES[t]))
    ms = some(M, K, 20)
    wy, oy, _, _ = blocks.rms_norm(host(total[ms]), host(w), 1e-6)
    within("y", y[ms], wy, oy + blocks.rounding(t == "bf16") * (np.abs(wy) + oy))
    for i in range(2):
        two, again = [x.clone(), res.clone()], nan(M, K, t=TYPES[t])
        B.fpq_rms_norm(*two, w, 1e-6, two[i], again)
        assert torch.equal(two[i], total) and torch.equal(again, y)
    ws = test_gpu_blocks.room(B.fpq_rms_norm_backward_workspace_size(M, K))
    gx, gw = nan(M, K, t=TYPES[t]), nan(K)
    B.fpq_rms_norm_backward(total, w, rstd, gy, gs, gx, gw, ws)
    wx, ox, _, _ = blocks.rms_norm_backward(host(total[ms]), host(w), host(rstd[ms]), host(gy[ms]), host(gs[ms]))
    within("grad_x", gx[ms], wx, ox + blocks.rounding(t == "bf16") * (np.abs(wx) + ox))
    for i in range(2):
        two, again = [gy.clone(), gs.clone()], nan(K)
        B.fpq_rms_norm_backward(total, w, rstd, *two, two[i], again, ws)
        assert torch.equal(two[i], gx) and torch.equal(again, gw)
