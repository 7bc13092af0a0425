"""Operators around the projections at values far out: NaN where codes are made, products near the ends of the range, infinities."""
import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2408_06995_amd import binding as B
from gpu_util import DEV
from test_gpu_blocks import E2M1, E4M3, TYPES, host, nan, quantize, room, rows, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("f", [E4M3, (5, 2, 15, 57344.0), (3, 4, 4, 0.0), (2, 1, 1, 0.0)])
@pytest.mark.parametrize("K", [64, 77, 6000])
def test_codes_of_norms_that_are_nan(K, f):
    """The codes are fpq_quantize's for the same values, of NaN with either sign too."""
    print(K, f, flush=True)
    x = rows(torch.Generator().manual_seed(K), 8, K, torch.float32)
    x.view(torch.int32)[2, 3], x.view(torch.int32)[4, K - 1], x[6, 5] = 0x7fc00000, 0xffc00000 - (1 << 32), float("inf")
    y, codes = nan(8, K), torch.full((8, B.fpq_padded_channels(K)), 0xee, dtype=torch.uint8, device=DEV)
    scale = torch.tensor([0.013], device=DEV)
    for w in (None, torch.linspace(-1, 1, K, device=DEV)):
        B.fpq_rms_norm(x, None, w, 1e-6, None, y, None, codes, f, None, scale)
        assert y[[2, 4]].isnan().all() and y[6, 5].isnan()
        want = torch.empty(B.fpq_code_bytes(8 * K, f[:3] + (f[3] or B.lib().fpq_format_max(*f[:3]),)), dtype=torch.uint8, device=DEV)
        B.fpq_quantize(y.view(-1), f, 0.0, scale, want)
        want = want.cpu().numpy()
        want = (want if want.size == 8 * K else blocks.unpack(want[None])).reshape(8, K)
        got = codes.cpu().numpy()
        assert np.array_equal(got[:, :K], want) and not got[:, K:].any()


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 16, 64, 70])
@pytest.mark.parametrize("x_exp,w_exp", [(125, -30), (120, -7), (-100, -30), (-60, -60), (-20, 100)])
def test_layers_whose_products_are_in_range(x_exp, w_exp, M, t):
    """Large x with small weights and the other way round: what is in range as a product counts in full."""
    print(x_exp, w_exp, M, t, flush=True)
    N, K = 40, 2000
    g = torch.Generator().manual_seed(M)
    codes, scales = quantize(rows(g, N, K, torch.float32), E2M1)
    scales.fill_(127 + w_exp)
    x = torch.rand(M, K, generator=g) + 0.5
    x[:, 1::2] *= -1
    x = torch.ldexp(x.double(), torch.tensor(x_exp)).to(TYPES[t]).to(DEV)
    wv = blocks.block_values(blocks.unpack(codes.cpu().numpy()), scales.cpu().numpy(), 4, K)
    y = nan(M, N, t=TYPES[t])
    B.fpq_block_linear(x, codes, scales, None, y, room(B.fpq_block_linear_workspace_size(M, N, K, int(t == "bf16"))))
    within("y", y, *blocks.block_linear(host(x), wv, None, t == "bf16"))


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M", [2, 4, 5, 16, 40, 70])
def test_infinities_stay_in_their_rows(M, t):
    """A row of x with an infinity or NaN has no finite result and no other row is touched; grad_bias, grad_x and grad_w of such a row the same."""
    print(M, t, flush=True)
    N, K = 48, 96
    g = torch.Generator().manual_seed(M)
    codes, scales = quantize(rows(g, N, K, torch.float32).clamp(min=0.1), E2M1)              # (no zeros among them)
    x, gy, w = rows(g, M, K, TYPES[t]), rows(g, M, N, TYPES[t]), rows(g, N, K, TYPES[t])
    ty = int(t == "bf16")
    for bad in (float("inf"), -float("inf"), float("nan")):
        a, b = x.clone(), gy.clone()
        a[1, 37], b[1, 11] = bad, bad
        y = nan(M, N, t=TYPES[t])
        B.fpq_block_linear(a, codes, scales, None, y, room(B.fpq_block_linear_workspace_size(M, N, K, ty)))
        finite = y.isfinite().all(1).cpu()
        assert not y[1].isfinite().any() and finite.sum() == M - 1
        gx, gw, gb = nan(M, K, t=TYPES[t]), nan(N, K, t=TYPES[t]), nan(N)
        for out in ((gx, gw, gb), (None, None, gb), (gx, None, None), (None, gw, gb)):
            for o in out:
                if o is not None:
                    o.zero_()
            B.fpq_linear_backward(x, None, w, b, *out, room(B.fpq_linear_backward_workspace_size(M, N, K, ty)))
            if out[0] is not None:
                assert not gx[1].isfinite().any() and gx.isfinite().all(1).sum() == M - 1
            if out[1] is not None:
                assert not gw[11].isfinite().any() and gw.isfinite().all(1).sum() == N - 1
            if out[2] is not None:
                assert not gb[11].isfinite() and gb.isfinite().sum() == N - 1
