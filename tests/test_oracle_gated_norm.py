"""The check of bf16 gated gradients in norm (oracle/blocks.py: gated_spread), held against an emulation of their roundings in 64 bits: what the
kernels' roundings give passes, a mistake planted in the emulation does not."""
import numpy as np
import pytest

from oracle import adapt, blocks
from test_oracle_attention_norm import planes


def emulate(x, w, a, g, act, gh, operand_planes=2, fault=None):
    f, slope, _, _ = blocks.gate(g, act)
    d = np.concatenate([gh * f, gh * a * slope], 1)
    d = planes(d, operand_planes)
    if fault == "a row of dg":
        d[1, d.shape[1] // 2:] = 0
    return [adapt.bf16(v) * (0.98 if fault == "2 percent" else 1.0) for v in (d @ w, d.T @ x)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,N,K", [(300, 160, 320), (257, 96, 160), (64, 200, 128), (500, 77, 65)])
def test_mistakes_are_outside_and_roundings_are_not(M, N, K, act):
    rng = np.random.default_rng(M + N + K)
    x, a, g, gh = (adapt.bf16(rng.standard_normal(s)) for s in ((M, K), (M, N), (M, N), (M, N)))
    w = adapt.bf16(rng.standard_normal((2 * N, K)) * K ** -0.5)
    want = [v for v, _ in blocks.gated_backward(x, w, a, g, act, gh, True)[:2]]
    spread = blocks.gated_spread(x, w, a, g, act, gh)
    far = lambda **how: [adapt.off_in_norm(got, v, s) for got, v, s in zip(emulate(x, w, a, g, act, gh, **how), want, spread)]
    assert all(f <= 1 for f in far()), far()
    for how in (dict(operand_planes=1), dict(fault="2 percent"), dict(fault="a row of dg")):
        assert all(f > 1 for f in far(**how)), (how, far(**how))
