"""The norm on the residual stream and its gradient against the oracle, within the bounds that their roundings give."""
import numpy as np
import pytest
import torch

import oracle
from oracle import blocks
from paper_2408_06995_amd import binding as B
from gpu_util import DEV
from test_gpu_blocks import E4M3, TYPES, host, nan, room, rows, within

pytestmark = pytest.mark.gpu


def bytes_(*shape):
    return torch.full(shape, 0xee, dtype=torch.uint8, device=DEV)


def near_code(values, y, off, bits8_scale):
    """|values - y|: half a step of E4M3 in units of the scale, and what y itself is off."""
    s = bits8_scale
    return np.abs(values - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * s) + off * (1 + 2.0 ** -3) + 2.0 ** -20 * np.abs(y)


def check(M, K, t, ld=0, residual=True, weights=True, seed=1):
    g = torch.Generator().manual_seed(seed + M + K)
    bf16, t = t == "bf16", TYPES[t]
    wide = ld and K + ld
    x, res = rows(g, M, K, t, wide), rows(g, M, K, t, wide) if residual else None
    w = (1 + 0.3 * torch.randn(K, generator=g)).to(DEV) if weights else None
    total, y, rstd = nan(M, K + ld, t=t), nan(M, K + ld, t=t), nan(M)
    eps = 1e-6
    B.fpq_rms_norm(x, res, w, eps, total[:, :K], y[:, :K], rstd)
    r = (x.float() + res.float()).to(t) if residual else x
    assert torch.equal(total[:, :K], r) and total[:, K:].isnan().all() and y[:, K:].isnan().all()
    wv = host(w) if weights else np.ones(K)
    own = blocks.rounding(bf16)
    wy, oy, ws, os_ = blocks.rms_norm(host(r), wv, eps)
    within("y", y[:, :K], wy, oy + own * (np.abs(wy) + oy))
    within("rstd", rstd, ws, os_)
    # codes with a scale per tensor, and with one per block
    scale = float(np.abs(wy).max() / 300)
    codes = bytes_(M, B.fpq_padded_channels(K))
    B.fpq_rms_norm(x, res, w, eps, total[:, :K], None, None, codes, E4M3, scale)
    c = codes.cpu().numpy()
    assert not c[:, K:].any()
    v = oracle.dequantize(c[:, :K].copy(), E4M3, np.float32(scale)).astype(np.float64).reshape(M, K)
    assert near_code(v, wy, oy, scale).all()
    codes, scales = bytes_(M, blocks.padded(K)), bytes_(M, blocks.padded(K) // 32)
    B.fpq_rms_norm(x, res, w, eps, total[:, :K], None, None, codes, None, None, None, scales)
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    assert not c[:, K:].any()
    unit = np.repeat(2.0 ** (s.astype(float) - 127), 32, 1)[:, :K]
    assert near_code(blocks.block_values(c, s, 8, K), wy, oy, unit).all()
    top = np.abs(blocks._in_blocks(wy)).max(2)
    slack = blocks._in_blocks(oy).max(2)
    u = 2.0 ** (s.astype(float) - 127)
    assert np.all(top - slack <= 448 * u) and np.all(224 * u <= top + slack + (top == 0) * 224)
    # backward
    gy, gs = rows(g, M, K, t, wide), rows(g, M, K, t, wide)
    part = room(B.fpq_rms_norm_backward_workspace_size(M, K))
    for stream in (gs, None):
        gx, gw = nan(M, K + ld, t=t), nan(K)
        B.fpq_rms_norm_backward(total[:, :K], w, rstd, gy, stream, gx[:, :K], gw, part)
        wx, ox, ww, ow = blocks.rms_norm_backward(host(r), wv, host(rstd), host(gy), 0.0 if stream is None else host(stream))
        within("grad_x", gx[:, :K], wx, ox + own * (np.abs(wx) + ox))
        within("grad_w", gw, ww, ow + 2.0 ** -126)
        assert gx[:, K:].isnan().all()
    only, alone = nan(M, K, t=t), nan(K)
    B.fpq_rms_norm_backward(total[:, :K], w, rstd, gy, None, only, None, None)
    B.fpq_rms_norm_backward(total[:, :K], w, rstd, gy, None, None, alone, part)
    assert torch.equal(only, gx[:, :K]) and torch.equal(alone, gw)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 32), (3, 33), (5, 320), (2, 1280), (600, 64), (513, 320), (700, 1280), (520, 2048), (9, 4096), (3, 8192), (2, 8200), (2, 20000), (700, 77),
                                 (1025, 8)])
def test_sizes(M, K, t):
    print(M, K, t, flush=True)
    check(M, K, t)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K", [(4100, 128), (4101, 160), (2050, 256), (1700, 320), (1025, 512), (901, 640), (530, 1024), (451, 1280), (260, 2048), (231, 2560), (131, 4096),
                                 (121, 5120), (70, 8192), (61, 10240), (66000, 8)])
def test_many_rows(M, K, t):
    print(M, K, t, flush=True)
    check(M, K, t)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("residual,weights", [(False, True), (True, False), (False, False)])
def test_without_residual_or_weights(residual, weights, t):
    check(37, 160, t, 0, residual, weights)
    check(5, 131, t, 0, residual, weights)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("ld", [8, 3])
def test_strided_rows(ld, t):
    check(37, 160, t, ld)
    check(600, 333, t, ld)
    check(3, 10001, t, ld)


def test_in_place():
    """The stream may be updated where it is, and gradients written where they came from."""
    g = torch.Generator().manual_seed(3)
    x, res = rows(g, 40, 96, torch.bfloat16), rows(g, 40, 96, torch.bfloat16)
    total, y, rstd = nan(40, 96, t=torch.bfloat16), nan(40, 96, t=torch.bfloat16), nan(40)
    B.fpq_rms_norm(x, res, None, 1e-5, total, y, rstd)
    stream, y2 = res.clone(), nan(40, 96, t=torch.bfloat16)
    B.fpq_rms_norm(x, stream, None, 1e-5, stream, y2)
    assert torch.equal(stream, total) and torch.equal(y2, y)
    gy, gs = rows(g, 40, 96, torch.bfloat16), rows(g, 40, 96, torch.bfloat16)
    gx = nan(40, 96, t=torch.bfloat16)
    B.fpq_rms_norm_backward(total, None, rstd, gy, gs, gx, None)
    for at in (gy, gs):
        a, b = gy.clone(), gs.clone()
        to = a if at is gy else b
        B.fpq_rms_norm_backward(total, None, rstd, a, b, to, None)
        assert torch.equal(to, gx)


def test_other_formats_and_device_scale():
    g = torch.Generator().manual_seed(5)
    x = rows(g, 33, 80, torch.float32)
    y = nan(33, 80)
    B.fpq_rms_norm(x, None, None, 1e-6, None, y)
    for f in ((4, 3, 7, 448.0), (5, 2, 15, 57344.0), (3, 4, 4, 0.0), (2, 5, 2, 0.0), (4, 3, 8, 0.0), (2, 1, 1, 0.0)):
        codes, dev = bytes_(33, 80), torch.tensor([0.021], device=DEV)
        B.fpq_rms_norm(x, None, None, 1e-6, None, None, None, codes, f, None, dev)
        whole = f[:3] + (f[3] or B.lib().fpq_format_max(*f[:3]),)            # (the oracle takes the largest value, not a zero for it)
        want = oracle.quantize(y.cpu().numpy(), whole, np.float32(0.021))
        assert np.array_equal(codes.cpu().numpy(), want.reshape(33, 80)), f


def test_rows_with_infinities():
    g = torch.Generator().manual_seed(6)
    for t in TYPES.values():
        x = rows(g, 6, 72, t)
        x[2, 3], x[4, 70] = float("inf"), float("nan")
        y = nan(6, 72, t=t)
        B.fpq_rms_norm(x, None, None, 1e-6, None, y)
        keep = [0, 1, 3, 5]
        assert y[keep].isfinite().all() and y[4].isnan().all() and y[2, 3].isnan()
    z = torch.zeros(2, 64, device=DEV)
    B.fpq_rms_norm(z, None, None, 1e-6, None, z)
    assert not z.any()


def test_no_rows():
    e = torch.empty(0, 64, device=DEV)
    B.fpq_rms_norm(e, e, None, 1e-6, e, e, torch.empty(0, device=DEV))
    gw = nan(64)
    B.fpq_rms_norm_backward(e, None, torch.empty(0, device=DEV), e, None, e, gw, room(B.fpq_rms_norm_backward_workspace_size(0, 64)))
    assert not gw.any()
