"""Workspaces of gated calls of few rows, none for tokens and no room for packed weights where they are read in place; and of calls without rows."""
import pytest
import torch

from oracle import blocks
from paper_2408_06995_amd import binding as B


def test_sizes_of_few_rows():
    size = B.lib().fpq_gated_workspace_size
    for N, K in ((1, 1), (48, 40), (10240, 4096), (333, 1283)):
        for M in (1, 2, 15, 16):
            assert size(M, N, K, 0) == 0 and size(M, N, K, 1) == 0
        for M in (17, 33, 64):
            assert 0 < size(M, N, K, 0) <= 256
        assert size(65, N, K, 0) >= 65 * K * 6 + 2 * N * K * 6
    # bf16 above 16 rows: weights of more than 32 MB run in tiles, where odd rows of them are packed
    assert 0 < size(17, 1280, 5120, 1) <= 256 and size(17, 10240, 4097, 1) > 2 * 10240 * 4097 * 2


def test_sizes_without_rows():
    """Sums over no rows are zeros: the gradients have a workspace, the others none."""
    L = B.lib()
    for t in (0, 1):
        assert L.fpq_linear_backward_workspace_size(0, 48, 40, t) > 0 and L.fpq_gated_backward_workspace_size(0, 48, 40, t) > 0
        assert L.fpq_block_linear_workspace_size(0, 48, 40, t) == 0 and L.fpq_gated_workspace_size(0, 48, 40, t) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M", [1, 7, 16, 17, 40, 64])
def test_calls_with_no_more_than_the_stated_bytes(M, t):
    from gpu_util import DEV
    from test_gpu_blocks import host, nan, within
    from test_gpu_gated import Call
    c = Call(M, 96, 200, t)
    n = B.fpq_gated_workspace_size(M, c.N, c.K, int(c.bf16))
    ws = torch.full((n + 512,), 0xff, dtype=torch.uint8, device=DEV) if n else None
    h = nan(M, c.N, t=c.t)
    B.fpq_gated(c.x, c.w, c.bias, 0, h, None, None, None if ws is None else ws[:n])
    within("h", h, *blocks.gated(host(c.x), host(c.w), host(c.bias), "silu", c.bf16)[:2])
    assert ws is None or (ws[n:] == 0xff).all()
