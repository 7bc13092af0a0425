"""Attention and its gradient against the oracle in 64 bits, within the bounds that its roundings give."""
import numpy as np
import pytest
import torch

from oracle import adapt
from paper_2408_06995_amd import binding as B
from gpu_util import DEV

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def nan_like(t):
    return torch.full_like(t, float("nan"))


def room(n):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=DEV)


def tensors(B_, Lq, Lk, Hq, Hkv, D, t, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    q, go = (torch.randn(B_, Lq, Hq, D, generator=g) for _ in range(2))
    k, v = (torch.randn(B_, Lk, Hkv, D, generator=g) for _ in range(2))
    return [x.to(TYPES[t]).to(DEV) for x in (q * spread, k, v, go)]


def sizes(q, k):
    return (q.shape[0], q.shape[2], k.shape[2], q.shape[1], k.shape[1], q.shape[3], B.FPQ_TYPE_FP32 if q.dtype == torch.float32 else B.FPQ_TYPE_BF16)


def forward(q, k, v, scale, causal=0, lens=None, o=None):
    o = nan_like(q) if o is None else o
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), float("nan"), device=DEV)
    B.fpq_attention(q, k, v, o, lse, scale, causal, lens, room(B.fpq_attention_workspace_size(*sizes(q, k))))
    return o, lse


def backward(q, k, v, o, lse, go, scale, causal=0, lens=None, grads=None):
    grads = [nan_like(x) for x in (q, k, v)] if grads is None else grads
    B.fpq_attention_backward(q, k, v, o, lse, go, *grads, scale, causal, lens, room(B.fpq_attention_backward_workspace_size(*sizes(q, k))))
    return grads


def host(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def close(got, want, bound, what):
    got = host(got)
    assert np.array_equal(np.isneginf(want), np.isneginf(got)), what
    fine = np.isfinite(want)
    err = np.abs(got[fine] - want[fine])
    bad = ~(err <= bound[fine] + 1e-30)
    assert not bad.any(), "%s: %d of %d outside, worst %.3g of the bound" % (what, bad.sum(), bad.size, np.nanmax(err / (bound[fine] + 1e-30)))


def both(q, k, v, go, causal, lens, scale=None):
    scale = q.shape[3] ** -0.5 if scale is None else scale
    lens_t = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    o, lse = forward(q, k, v, scale, causal, lens_t)
    grads = backward(q, k, v, o, lse, go, scale, causal, lens_t)
    torch.cuda.synchronize()
    a = [host(x) for x in (q, k, v)]
    scale = float(np.float32(scale))
    want_o, want_lse = adapt.attention(*a, scale, causal, lens)
    want = adapt.attention_backward(*a, host(go), scale, causal, lens)
    to, tl, *tg = adapt.attention_bounds(*a, scale, causal, lens, q.dtype == torch.bfloat16, host(go))
    close(o, want_o, to, "o")
    close(lse, want_lse, tl, "lse")
    for name, got, w, t in zip(("gq", "gk", "gv"), grads, want, tg):
        close(got, w, t, name)


SHAPES = [  # samples, queries, keys, query heads, key heads, dimension
    (1, 1, 1, 1, 1, 8), (2, 1, 300, 4, 2, 64), (1, 64, 64, 8, 8, 160), (2, 130, 77, 2, 2, 40), (1, 33, 65, 6, 2, 80), (3, 5, 129, 2, 1, 128),
    (1, 257, 31, 1, 1, 96), (2, 100, 100, 2, 1, 48), (1, 128, 256, 1, 1, 32), (1, 31, 2000, 1, 1, 64),
]


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention(shape, causal, t):
    print(shape, causal, t, flush=True)
    q, k, v, go = tensors(*shape, t, 11)
    both(q, k, v, go, causal, None)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [1, 3, 7, 12, 17, 36, 50, 63, 79, 100, 129, 157])
def test_dimensions_off_the_alignment(dim, t):
    print(dim, t, flush=True)
    q, k, v, go = tensors(2, 37, 70, 2, 1, dim, t, dim)
    both(q, k, v, go, 1, [70, 33])


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("Lq,lens", [(40, [100, 0, 1, 39]), (1, [0, 64, 65, 1]), (150, [128, 129, 3, -5]), (64, [1000, 100, 99, 31])])
def test_lengths_of_samples(Lq, lens, causal, t):
    """Samples of no, one and all keys, lengths outside the buffer; what lies past a sample's keys is not used."""
    print(Lq, lens, causal, t, flush=True)
    q, k, v, go = tensors(4, Lq, 100, 4, 2, 64, t, 5)
    for b, n in enumerate(lens):
        k[b, max(0, min(n, 100)):] = float("nan")
        v[b, max(0, min(n, 100)):] = float("inf")
    both(q, k, v, go, causal, lens)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_many_rows_and_parts(t):
    """Several blocks of rows for several XCDs, and few rows over many keys, which are cut into parts."""
    q, k, v, go = tensors(3, 300, 300, 3, 3, 40, t, 21)
    both(q, k, v, go, 1, None)
    q, k, v, go = tensors(1, 3, 3000, 2, 1, 80, t, 22)
    assert B.fpq_attention_workspace_size(*sizes(q, k)) > 0
    both(q, k, v, go, 0, [2900])
    q, k, v, go = tensors(2, 1500, 9, 2, 2, 40, t, 23)
    assert B.fpq_attention_backward_workspace_size(*sizes(q, k)) > 2 * 1500 * 2 * 4 + 256
    both(q, k, v, go, 0, [9, 4])


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_large_scores(t):
    """Scores whose exponentials overflow without the running maximum, ascending and descending along the keys."""
    q, k, v, go = tensors(1, 70, 200, 2, 2, 32, t, 31, spread=12.0)
    both(q, k, v, go, 0, None, scale=1.0)
    k = (k.sum(-1, keepdim=True).sort(dim=1).values.expand_as(k) * 0.3).contiguous()
    both(q.abs().contiguous(), k, v, go, 1, None, scale=0.5)
    both(q.abs().contiguous(), -k, v, go, 0, None, scale=0.5)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_strides(t):
    """Columns of one projection's result, heads ahead of tokens, an offset of one element, gradients into such a layout."""
    D, Hq, Hkv, L = 40, 4, 2, 90
    g = torch.Generator().manual_seed(7)
    qkv = torch.randn(2, L, (Hq + 2 * Hkv) * D, generator=g).to(TYPES[t]).to(DEV)
    q, k, v = (x.unflatten(2, (-1, D)) for x in qkv.split([Hq * D, Hkv * D, Hkv * D], dim=2))
    go = torch.randn(2, Hq, L, D, generator=g).to(TYPES[t]).to(DEV).transpose(1, 2)
    both(q, k, v, go, 1, None)
    flat = torch.zeros(q.numel() + 1, dtype=q.dtype, device=DEV)
    off = flat[1:].view(q.shape)
    off.copy_(q)
    both(off, k, v, go, 1, None)
    o, lse = forward(q, k, v, 0.2, 1)
    grads = backward(q, k, v, o, lse, go, 0.2, 1)
    wide = torch.full_like(qkv, float("nan"))
    parts = [x.unflatten(2, (-1, D)) for x in wide.split([Hq * D, Hkv * D, Hkv * D], dim=2)]
    backward(q, k, v, o, lse, go, 0.2, 1, grads=parts)
    for a, b in zip(grads, parts):
        assert torch.equal(a, b)
    other = torch.full((2, Hq, L, D + 3), float("nan"), dtype=q.dtype, device=DEV)
    o2, _ = forward(q, k, v, 0.2, 1, o=other[..., :D].transpose(1, 2))
    assert torch.equal(o, o2) and torch.isnan(other[..., D:]).all()
    shared = k[:, :, :1].expand(-1, -1, Hkv, -1)                      # one key head seen as several: a stride of zero
    assert torch.equal(forward(q, shared, v, 0.2)[0], forward(q, shared.contiguous(), v, 0.2)[0])


def test_bits_repeat():
    for t in TYPES:
        q, k, v, go = tensors(2, 333, 333, 4, 2, 64, t, 41)
        first = None
        for _ in range(3):
            o, lse = forward(q, k, v, 0.125, 1)
            now = [o, lse] + backward(q, k, v, o, lse, go, 0.125, 1)
            assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
            first = now


def test_no_keys_and_no_queries():
    q, k, v, go = tensors(2, 9, 4, 2, 2, 16, "fp32", 51)
    o, lse = forward(q, k[:, :0], v[:, :0], 1.0)
    assert torch.all(o == 0) and torch.all(torch.isneginf(lse))
    gq, gk, gv = backward(q, k[:, :0], v[:, :0], o, lse, go, 1.0)
    assert torch.all(gq == 0) and gk.numel() == 0
    o, lse = forward(q[:, :0], k, v, 1.0)
    gq, gk, gv = backward(q[:, :0], k, v, o, lse, go[:, :0], 1.0)
    assert torch.all(gk == 0) and torch.all(gv == 0)


def test_a_value_that_is_no_number_reaches_the_rows_that_see_it():
    for t in TYPES:
        q, k, v, go = tensors(2, 40, 40, 2, 2, 32, t, 61)
        k[0, 7, 1, 3] = float("nan")
        o, lse = forward(q, k, v, 0.2)
        assert torch.isnan(o[0, :, 1]).all() and torch.isnan(lse[0, 1]).all()
        assert torch.isfinite(o[0, :, 0]).all() and torch.isfinite(o[1]).all() and torch.isfinite(lse[1]).all()


def test_another_stream_and_a_graph():
    q, k, v, go = tensors(1, 200, 200, 2, 2, 64, "bf16", 71)
    o, lse = forward(q, k, v, 0.125, 1)
    grads = backward(q, k, v, o, lse, go, 0.125, 1)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    bufs = [nan_like(x) for x in (o, lse, *grads)]
    ws = room(max(B.fpq_attention_workspace_size(*sizes(q, k)), B.fpq_attention_backward_workspace_size(*sizes(q, k))))

    def call():
        B.fpq_attention(q, k, v, bufs[0], bufs[1], 0.125, 1, None, ws)
        B.fpq_attention_backward(q, k, v, bufs[0], bufs[1], go, *bufs[2:], 0.125, 1, None, ws)

    with torch.cuda.stream(s):
        call()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(bufs, (o, lse, *grads)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for x in bufs:
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bufs, (o, lse, *grads)))


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("shape", [(32, 300, 77, 8, 8, 40), (64, 270, 33, 8, 4, 64), (128, 257, 96, 2, 2, 80), (128, 260, 1, 2, 2, 96), (128, 300, 95, 2, 2, 33),
                                   (128, 257, 64, 2, 2, 128), (128, 257, 70, 2, 2, 160), (256, 513, 32, 1, 1, 8)])
def test_few_keys_of_many_rows(shape, causal, t):
    """Many blocks of rows over a tile or two of keys; samples of fewer keys and of none, with others' values behind."""
    print(shape, causal, t, flush=True)
    q, k, v, go = tensors(*shape, t, 41)
    n = shape[2]
    lens = [(7 * b) % (n + 1) if b % 3 else n for b in range(shape[0])]
    for b in range(shape[0]):
        k[b, lens[b]:] = float("nan")
        v[b, lens[b]:] = float("inf")
    scale = shape[5] ** -0.5
    o, lse = forward(q, k, v, scale, causal, torch.tensor(lens, dtype=torch.int32, device=DEV))
    few = sorted({0, 1, 2, shape[0] - 1, *(b for b in range(shape[0]) if lens[b] == 0)})[:6]        # samples are independent
    a = [host(x[few]) for x in (q, k, v)]
    some = [lens[b] for b in few]
    scale = float(np.float32(scale))
    want_o, want_lse = adapt.attention(*a, scale, causal, some)
    to, tl = adapt.attention_bounds(*a, scale, causal, some, t == "bf16")[:2]
    close(o[few], want_o, to, "o")
    close(lse[few], want_lse, tl, "lse")
    assert not o.isnan().any() and not lse.isnan().any()


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("dim", [40, 64, 80, 96, 128, 157, 160])
@pytest.mark.parametrize("shape", [(32, 150, 140, 8, 4), (3, 640, 500, 4, 2), (6, 200, 333, 8, 1)])
def test_larger_problems(shape, dim, causal, t):
    """Workgroups of two and four wavefronts, one plane of the probabilities in bf16, blocks of one head's rows, samples of different
    lengths and of none; a few of the samples against the oracle, which they are independent of."""
    print(shape, dim, causal, t, flush=True)
    n = shape[2]
    lens = [(37 * b + 5) % (n + 1) if b % 3 else n for b in range(shape[0])]
    lens[1] = 0
    q, k, v, go = tensors(*shape, dim, t, dim)
    for b in range(shape[0]):
        k[b, lens[b]:] = float("nan")
        v[b, lens[b]:] = float("inf")
    scale = dim ** -0.5
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    o, lse = forward(q, k, v, scale, causal, lens_t)
    grads = backward(q, k, v, o, lse, go, scale, causal, lens_t)
    few = [0, 1, shape[0] - 1]
    a = [host(x[few]) for x in (q, k, v)]
    some = [lens[b] for b in few]
    scale = float(np.float32(scale))
    want_o, want_lse = adapt.attention(*a, scale, causal, some)
    want = adapt.attention_backward(*a, host(go[few]), scale, causal, some)
    to, tl, *tg = adapt.attention_bounds(*a, scale, causal, some, t == "bf16", host(go[few]))
    close(o[few], want_o, to, "o")
    close(lse[few], want_lse, tl, "lse")
    for name, got, w, b in zip(("gq", "gk", "gv"), grads, want, tg):
        close(got[few], w, b, name)
    assert not any(x.isnan().any() for x in (o, lse, *grads))
