"""Sums of a bias's gradient over many rows, made beside the weights' gradient: values of one sign that are the same in every row, as a mean's gradient
gives them, whose roundings go the same way."""
import pytest
import torch

from paper_2408_06995_amd import binding as B
from gpu_util import DEV
from test_gpu_blocks import E4M3, TYPES, quantize, room

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


@pytest.mark.parametrize("kept", [False, True], ids=["x", "blocks"])
@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M", [4097, 1 << 18, (1 << 22) + 33])
def test_equal_rows(M, t, kept):
    """A lane adds up 16 steps, 384 pairs at the most, then these sums, three planes of M / 64 steps over the slices (27 where one tile has this many
    steps), then the slices: twice 384 roundings of pairs, 3 M / (16 64 27) of the former and 64 for the rest, each of 2^-24 of a sum that only grows."""
    print(M, t, kept, flush=True)
    N, K = 64, 32
    gy = (torch.rand(N, generator=torch.Generator().manual_seed(M)) + 0.5).to(TYPES[t]).to(DEV).expand(M, N).contiguous()
    x = torch.ones(M, K, dtype=TYPES[t], device=DEV)
    w = torch.ones(N, K, dtype=TYPES[t], device=DEV)
    x, scales = quantize(x, E4M3) if kept else (x, None)
    want = gy[0].double() * M
    ws = room(B.fpq_linear_backward_workspace_size(M, N, K, int(t == "bf16")))
    for gx in (None, torch.empty(M, K, dtype=TYPES[t], device=DEV)):
        gw, gb = torch.empty_like(w), torch.empty(N, device=DEV)
        B.fpq_linear_backward(x, scales, w, gy, gx, gw, gb, ws)
        off = ((gb.double() - want).abs() / want).max().item()
        most = (2 * 384 + 3 * M // (16 * 64 * 27) + 64) * U32
        print("off %.3g of %.3g" % (off, most), flush=True)
        assert off <= most
