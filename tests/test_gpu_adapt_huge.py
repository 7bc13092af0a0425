"""Tensors of more than 2^31 elements in the operators for adapting a model, and calls side by side on two streams."""
import pytest
import torch

from paper_2408_06995_amd import binding as B
from gpu_util import DEV
from test_gpu_attention import backward, forward, nan_like, room, sizes, tensors
from test_gpu_adapter import Call

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("samples,keys", [(1, (1 << 24) + 1001), (3, (1 << 23) + 5)])
def test_attention_over_keys_past_32_bit_offsets(samples, keys, t):
    """One token whose two keys that count are the first and the last of the cache."""
    print(samples, keys, t, flush=True)
    D = 128
    g = torch.Generator().manual_seed(3)
    q = torch.ones(samples, 1, 1, D, dtype=TYPES[t], device=DEV)
    k, v = (torch.zeros(samples, keys, 1, D, dtype=TYPES[t], device=DEV) for _ in range(2))
    ends = torch.randint(-4, 5, (samples, 2, 1, D), generator=g).to(TYPES[t]).to(DEV)
    go = torch.randint(-4, 5, (samples, 1, 1, D), generator=g).to(TYPES[t]).to(DEV)
    for i, at in enumerate((0, -1)):
        k[:, at] = 1.0
        v[:, at] = ends[:, i]
    assert k.numel() > 1 << 31
    # scores: 128 for the two, 0 for the rest, whose weight e^-128 keys is below every rounding here
    o, lse = forward(q, k, v, 1.0)
    assert torch.equal(o[:, 0].float(), ends.float().mean(1))
    assert torch.all((lse - 128.6931471805599453).abs() <= 4 * 2.0 ** -24 * 129)
    gq, gk, gv = backward(q, k, v, o, lse, go, 1.0)
    # p = 1/2 each (its log-sum is off by at most 2^-17), ds = p (dp - delta)
    dp = (ends.float() * go.float()).sum(-1)[:, :, 0]
    delta = dp.mean(1, keepdim=True)
    ds = 0.5 * (dp - delta)
    near = lambda a, b: bool(((a.float() - b).abs() <= 2.0 ** -7 * b.abs() + 2.0 ** -13).all())
    for i, at in enumerate((0, -1)):
        assert near(gv[:, at, 0], 0.5 * go[:, 0, 0].float()) and near(gk[:, at, 0], ds[:, i, None].expand(-1, D))
    assert near(gq[:, 0, 0], ds.sum(1, keepdim=True).expand(-1, D))
    for x in (gk, gv):
        assert float(x[:, 1:-1].abs().max()) < 1e-30


@pytest.mark.parametrize("x,w", [("fp32", "bf16"), ("bf16", "bf16")])
def test_adapters_of_rows_past_32_bit_offsets(x, w):
    """The last rows are those of a request of their own: what a call for them alone gives, in whole numbers."""
    print(x, w, flush=True)
    M, tail, K, N, R = (1 << 25) + 77, 200, 72, 80, 8
    g = torch.Generator(device=DEV).manual_seed(4)
    ints = lambda *s: torch.randint(-2, 3, s, generator=g, device=DEV, dtype=torch.int8)
    small = Call(tail, N, K, R, [0, tail], [1], 2, x, w)
    large = Call(64, N, K, R, [0, 0], [0], 2, x, w)
    small.a, small.b = (ints(*t.shape).to(t.dtype) for t in (small.a, small.b))
    small.scaling = torch.tensor([1.0, 2.0], device=DEV)
    large.a, large.b, large.scaling = small.a, small.b, small.scaling
    for n, c in (("x", K), ("base", N), ("gy", N), ("gx_base", K)):
        big = torch.empty(M, c, dtype=TYPES[x], device=DEV)
        for lo in range(0, M, 1 << 22):
            big[lo:lo + (1 << 22)] = ints(min(1 << 22, M - lo), c)
        setattr(large, n, big)
        setattr(small, n, big[M - tail:].clone())
    large.starts = torch.tensor([0, M - tail, M], dtype=torch.int32, device=DEV)
    large.of = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    large.sizes = (M, N, K, R, 2, 2)
    large.shared = (large.x, large.a, large.b, large.scaling, large.starts, large.of)
    assert large.x.numel() > 1 << 31
    y, t = large.forward()
    sy, st = small.forward()
    assert torch.equal(y[M - tail:], sy) and torch.equal(t[M - tail:], st)
    gx, ga, gb = large.backward(t)
    sgx, sga, sgb = small.backward(st)
    assert torch.equal(gx[M - tail:], sgx) and torch.equal(ga[1], sga[1]) and torch.equal(gb[1], sgb[1])
    # and rows in the middle, past half of 2^31 elements
    lo = (1 << 24) + 12345
    rows = slice(lo, lo + 100)
    T = large.x[rows].float() @ large.a[0].float().T
    assert torch.equal(t[rows], T) and torch.equal(y[rows], (large.base[rows].float() + T @ large.b[0].float().T).to(y.dtype))


def test_adamw_of_the_most_elements():
    n, tail = (1 << 31) - 1, 2047                    # (seven blocks of 256 and one of 255)
    g = torch.Generator(device=DEV).manual_seed(5)
    param, grad = (torch.zeros(n, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    scales = [torch.ones((n + 255) // 256, device=DEV) for _ in range(2)]
    for t, s in ((param, 0.1), (grad, 0.01)):
        t[n - tail:] = (torch.randn(tail, generator=g, device=DEV) * s).bfloat16()
        t[:tail] = t[n - tail:]
    small = [t[n - tail:].clone() for t in (param, grad, m, v)] + [torch.ones(8, device=DEV) for _ in range(2)]
    for items in ((param, grad, m, v, *scales, None), (*small, None)):
        arr = B.adamw_tensors([items])
        plan = torch.empty(B.fpq_adamw_plan_size(arr), dtype=torch.uint8, device=DEV)
        pieces = B.fpq_adamw_plan(arr, plan)
        for step in (1, 2):
            B.fpq_adamw_step(plan, pieces, 1e-3, 0.9, 0.99, 1e-8, 0.1, step)
    torch.cuda.synchronize()
    for big, little in zip((param, grad, m, v), small):
        assert torch.equal(big[n - tail:], little) and torch.equal(big[:tail - 255], little[:tail - 255])
    for big, little in zip(scales, small[4:]):
        assert torch.equal(big[-8:], little)
    assert not param[tail:n - tail].any() and not m[tail:n - tail].any()


def test_two_streams_at_once():
    """Calls of all operators on two streams, with workspaces of their own, while the other stream's are under way."""
    def job(seed):
        q, k, v, go = tensors(2, 700, 650, 4, 2, 64, ["fp32", "bf16"][seed], 60 + seed)
        c = Call(3000, 160, 320, 16, [0, 1234, 3000], [1, 0], 2, "fp32", "bf16", seed=70 + seed)
        ws = [room(n) for n in (B.fpq_attention_workspace_size(*sizes(q, k)), B.fpq_attention_backward_workspace_size(*sizes(q, k)),
                                B.fpq_adapter_workspace_size(*c.sizes), B.fpq_adapter_backward_workspace_size(*c.sizes))]
        out = [nan_like(q), torch.empty(2, 4, 700, device=DEV), nan_like(q), nan_like(k), nan_like(v), nan_like(c.base), torch.empty(3000, 16, device=DEV), nan_like(c.x),
               torch.empty(c.a.shape, device=DEV), torch.empty(c.b.shape, device=DEV)]

        def call():
            B.fpq_attention(q, k, v, *out[:2], 0.125, 1, None, ws[0])
            B.fpq_adapter_apply(*c.shared, c.base, *out[5:7], ws[2])
            B.fpq_attention_backward(q, k, v, *out[:2], go, *out[2:5], 0.125, 1, None, ws[1])
            B.fpq_adapter_backward(*c.shared, out[6], c.gy, c.gx_base, *out[7:], ws[3])
        return call, out

    jobs = [job(0), job(1)]
    want = []
    for call, out in jobs:
        call()
        torch.cuda.synchronize()
        want.append([x.clone() for x in out])
        for x in out:
            x.fill_(float("nan"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        for s, (call, _) in zip(streams, jobs):
            with torch.cuda.stream(s):
                call()
    torch.cuda.synchronize()
    for (_, out), w in zip(jobs, want):
        assert all(torch.equal(a, b) for a, b in zip(out, w))
