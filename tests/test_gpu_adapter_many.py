"""Adapters of very many requests: each row gets its request's adapter, whatever the runs of rows between."""
import numpy as np
import pytest
import torch

from paper_2408_06995_amd import binding as B
from gpu_util import DEV
from test_gpu_adapter import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x,w", [("fp32", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("requests", [61, 62, 63, 126, 4000, 4097, 9000])
def test_requests_around_the_rounds_of_the_search(requests, x, w):
    """Requests of no row, of one, and of more than a tile; rows of no request ahead and behind."""
    print(requests, x, w, flush=True)
    rng = np.random.default_rng(requests)
    lengths = np.where(rng.random(requests) < 0.01, 75, rng.integers(0, 3, requests))
    starts = (5 + np.concatenate([[0], np.cumsum(lengths)])).tolist()
    Call(starts[-1] + 7, 40, 24, 8, starts, rng.integers(-1, 6, requests).tolist(), 5, x, w, seed=requests).check()


def test_as_many_requests_as_are_accepted():
    """2^21 requests of nought to three rows, against the same rows gathered by adapter in 64 bits."""
    n, adapters, K, N, R = 1 << 21, 3, 8, 8, 4
    g = torch.Generator(device=DEV).manual_seed(1)
    lengths = torch.randint(0, 4, (n,), generator=g, device=DEV)
    starts = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), lengths.cumsum(0)])
    M = int(starts[-1])
    of = torch.randint(-1, adapters, (n,), generator=g, device=DEV)
    x, base, gy = (torch.randint(-3, 4, (M, c), generator=g, device=DEV).float() for c in (K, N, N))
    a, b = (torch.randint(-3, 4, s, generator=g, device=DEV).float() for s in ((adapters, R, K), (adapters, N, R)))
    scaling = torch.tensor([1.0, 2.0, 4.0], device=DEV)
    y, t, gx = torch.empty_like(base), torch.empty(M, R, device=DEV), torch.empty_like(x)
    ga, gb = torch.empty_like(a), torch.empty_like(b)
    ws = torch.empty(B.fpq_adapter_backward_workspace_size(M, N, K, R, n, adapters), dtype=torch.uint8, device=DEV)
    shared = (x, a, b, scaling, starts.int(), of.int())
    B.fpq_adapter_apply(*shared, base, y, t)
    print("forward", flush=True)
    B.fpq_adapter_backward(*shared, t, gy, None, gx, ga, gb, ws)
    torch.cuda.synchronize()
    print("backward", flush=True)
    mine = torch.repeat_interleave(of, lengths, output_size=M)
    assert torch.equal(y[mine < 0], base[mine < 0]) and torch.all(t[mine < 0] == 0) and torch.all(gx[mine < 0] == 0)
    for i in range(adapters):
        # whole numbers: every product and every sum is exact, but for the rows' sums of the gradients, which pass 2^24
        rows, s = mine == i, float(scaling[i])
        X, G, A, Bt = x[rows].double(), gy[rows].double(), a[i].double(), b[i].double()
        T = (X[:, None, :] * A).sum(2)
        dT = s * (G[:, :, None] * Bt).sum(1)
        assert torch.equal(t[rows].double(), T) and torch.equal(y[rows].double(), base[rows].double() + s * (T[:, None, :] * Bt).sum(2))
        assert torch.equal(gx[rows].double(), (dT[:, :, None] * A).sum(1))
        for got, l, r in ((ga[i], dT, X), (gb[i], s * G, T)):
            want = torch.stack([(l * r[:, k:k + 1]).sum(0) for k in range(r.shape[1])], 1)
            mass = torch.stack([(l * r[:, k:k + 1]).abs().sum(0) for k in range(r.shape[1])], 1)
            # one rounding of a partial sum, at most the sum of its terms' magnitudes, per term
            assert torch.all((got.double() - want).abs() <= 2.0 ** -24 * mass * rows.sum())
