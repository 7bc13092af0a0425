"""bf16 attention and its gradient in norm: no further from the rounded result in 64 bits than the roundings of the operands and of o
make them, per output and per head, whatever else is in the call."""
import numpy as np
import pytest
import torch

from oracle import adapt
from test_gpu_attention import backward, forward, host, tensors

pytestmark = pytest.mark.gpu

NAMES = ("o", "gq", "gk", "gv")


def near(results, q, k, v, go, scale, causal, lens, samples):
    """`results` of the whole call, of which `samples` are compared."""
    a = [host(x[samples]) for x in (q, k, v, go)]
    lens = None if lens is None else [lens[b] for b in samples]
    scale = float(np.float32(scale))
    want = (adapt.attention(*a[:3], scale, causal, lens)[0], *adapt.attention_backward(*a, scale, causal, lens))
    spread = adapt.attention_spread(*a[:3], scale, causal, lens, a[3])
    far = {}
    for name, got, w, s in zip(NAMES, results, want, spread):
        got = host(got[samples])
        for h in range(w.shape[2]):
            far[name, h] = adapt.off_in_norm(got[:, :, h], w[:, :, h], s[:, :, h])
    print({name: "%.3f" % max(f for (n, _), f in far.items() if n == name) for name in NAMES}, flush=True)
    assert all(f <= 1 for f in far.values()), {k: f for k, f in far.items() if not f <= 1}


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("shape,samples", [
    ((1, 300, 300, 4, 2, 64), [0]), ((2, 150, 140, 8, 4, 128), [0, 1]), ((3, 640, 500, 4, 2, 128), [0, 2]), ((6, 200, 333, 8, 1, 160), [5]),
    ((3, 640, 500, 4, 2, 157), [1]), ((32, 150, 140, 8, 4, 160), [31]), ((128, 257, 96, 2, 2, 80), [0, 127]), ((8, 1000, 77, 8, 8, 40), [7]),
    ((4, 64, 95, 4, 4, 40), [0, 3]), ((2, 2048, 300, 8, 8, 96), [1]),
])
def test_no_further_than_the_roundings(shape, samples, causal):
    print(shape, causal, flush=True)
    q, k, v, go = tensors(*shape, "bf16", 83)
    scale = shape[5] ** -0.5
    o, lse = forward(q, k, v, scale, causal)
    near([o, *backward(q, k, v, o, lse, go, scale, causal)], q, k, v, go, scale, causal, None, samples)


@pytest.mark.parametrize("Lq,Lk,D", [(24, 95, 40), (100, 100, 64), (64, 64, 160), (1, 300, 128)])
def test_a_sample_alone_and_among_many(Lq, Lk, D):
    """The precision of a sample's results is the same in a call of its own and in one of 128 samples."""
    q, k, v, go = tensors(128, Lq, Lk, 4, 4, D, "bf16", 85)
    scale = D ** -0.5
    for part in (slice(0, 128), slice(0, 1)):
        x = [t[part].contiguous() for t in (q, k, v, go)]
        o, lse = forward(*x[:3], scale)
        print(Lq, Lk, D, part, flush=True)
        near([o, *backward(*x[:3], o, lse, x[3], scale)], *x, scale, False, None, [0])
