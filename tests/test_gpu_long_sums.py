"""Sums over many rows, beside the weights' gradient or in a pass of their own: values of one sign that are the same in every row, as a mean's gradient gives
them, whose roundings go the same way."""
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
    steps), then the slices: twice 384 roundings of pairs, 3 M / (16 64 27) of the former and 64 for the rest, each of 2^-24 of a sum that only grows.  Where the
    sums have a pass of their own instead (fp32 from x in its type, in tiles of one plane), a lane adds up M / 2048 rows, and 64 for the parts."""
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
        most = max(2 * 384 + 3 * M // (16 * 64 * 27) + 64, M // 2048 + 64) * U32
        print("off %.3g of %.3g" % (off, most), flush=True)
        assert off <= most


@pytest.fixture
def give_back():
    yield
    torch.cuda.empty_cache()


def off_by(got, want):
    off = ((got.double() - want).abs() / want.abs()).max().item()
    print("off %.3g" % off, flush=True)
    return off


def test_passes_over_many_rows(give_back):
    """Sums that have a pass of their own: a lane adds up 2048 rows, the second launch a sixteenth of at most 32768 parts.  The values are 1.1 or so, so that
    none is a whole number of units in the last place of the sum."""
    M, N = (1 << 26) + 77, 8
    most = (2048 + (1 << 26) // 8192 // 16 + 32) * U32
    value = torch.linspace(1.1, 1.9, N, device=DEV)
    gy = value.expand(M, N).contiguous()
    gb = torch.empty(N, device=DEV)
    B.fpq_linear_backward(None, None, torch.empty(N, 8, device=DEV), gy, None, None, gb, room(B.fpq_linear_backward_workspace_size(M, N, 8, 0)))
    assert off_by(gb, value.double() * M) <= most
    # the norm's weights: gy r rstd with r of one and rstd of one
    one, gw = torch.ones(M, N, device=DEV), torch.empty(N, device=DEV)
    B.fpq_rms_norm_backward(one, None, one.view(-1)[:M], gy, None, None, gw, room(B.fpq_rms_norm_backward_workspace_size(M, N)))
    assert off_by(gw, value.double() * M) <= most
    del one
    # a of one, a gate of 1.25: da = gh silu(1.25), dg = gh silu'(1.25), as they come out for few rows
    pre, x, w = torch.ones(M, 2 * N, device=DEV), torch.empty(M, 1, device=DEV), torch.empty(2 * N, 1, device=DEV)
    pre[:, N:] = 1.25
    gb, few = torch.empty(2 * N, device=DEV), torch.empty(2 * N, device=DEV)
    for m, out in ((1, few), (M, gb)):
        B.fpq_gated_backward(None, None, w, pre[:m], None, B.FPQ_GATE_SILU, gy[:m], None, None, out, room(B.fpq_gated_backward_workspace_size(m, N, 1, 0)))
    assert off_by(gb, few.double() * M) <= most
