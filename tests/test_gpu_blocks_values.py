"""Operators around the projections at values far out: NaN where codes are made."""
import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2408_06995_amd import binding as B
from gpu_util import DEV
from test_gpu_blocks import E4M3, nan, rows

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
