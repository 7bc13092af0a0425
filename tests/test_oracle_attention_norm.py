"""The check of bf16 attention in norm (oracle/adapt.py: attention_spread, off_in_norm), held against an emulation of its roundings
in 64 bits: what the kernels' roundings give passes, a mistake planted in the emulation does not."""
import numpy as np
import pytest

from oracle import adapt


def planes(x, n):
    """x as the sum of n bf16 values, each the rest's rounding."""
    out, rest = np.zeros_like(x), x
    for _ in range(n):
        out, rest = out + adapt.bf16(rest), rest - adapt.bf16(rest)
    return out


def emulate(q, k, v, go, scale, causal, operand_planes=2, fault=None):
    o, gq, gk, gv = np.zeros(q.shape), np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    G, n = q.shape[2] // k.shape[2], k.shape[1]
    for b in range(q.shape[0]):
        for x in range(q.shape[2]):
            Q, K, V, dO = q[b, :, x], k[b, :, x // G], v[b, :, x // G], go[b, :, x]
            see = adapt.visible(len(Q), n, causal)
            s = np.where(see, scale * (Q @ K.T), -np.inf)
            top = np.maximum(s.max(1, keepdims=True), -1e30)
            e = np.exp(s - top)
            p = e / np.maximum(e.sum(1, keepdims=True), 1e-300)
            o[b, :, x] = adapt.bf16(planes(p, operand_planes) @ V)
            dp = dO @ V.T
            delta = (dO * o[b, :, x]).sum(1, keepdims=True) * {"no delta": 0.0, "half of delta": 0.5}.get(fault, 1.0)
            p_in, ds_in = planes(p, operand_planes), planes(p * (dp - delta), operand_planes)
            gq[b, :, x] = scale * (ds_in @ K)
            rows = np.arange(len(Q))
            kept = (rows < len(Q) - 40) | (rows >= len(Q) - 8) if fault == "a tile of queries" else rows >= 0
            gk[b, :, x // G] += scale * (ds_in[kept].T @ Q[kept])
            gv[b, :, x // G] += p_in[kept].T @ dO[kept]
    if fault == "gk times 0.9":
        gk *= 0.9
    return o, adapt.bf16(gq), adapt.bf16(gk), adapt.bf16(gv)


#: What each mistake makes wrong.
FAULTS = {"gk times 0.9": ["gk"], "no delta": ["gq", "gk"], "half of delta": ["gq", "gk"], "a tile of queries": ["gk", "gv"], "one plane": ["o"]}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(1, 300, 300, 4, 2, 64), (2, 150, 140, 8, 4, 128), (1, 640, 500, 4, 2, 128), (1, 200, 333, 8, 1, 160),
                                   (1, 640, 500, 4, 2, 157), (2, 257, 96, 2, 2, 80), (1, 300, 77, 4, 4, 40), (4, 64, 95, 4, 4, 40), (1, 150, 140, 8, 4, 160),
                                   (1, 1000, 77, 8, 8, 40), (1, 2048, 300, 8, 8, 96), (1, 24, 95, 4, 4, 40), (1, 100, 100, 4, 4, 64), (1, 64, 64, 4, 4, 160)])
def test_mistakes_are_outside_and_roundings_are_not(shape, causal):
    B, Lq, Lk, Hq, Hkv, D = shape
    rng = np.random.default_rng(sum(shape))
    q, go = (adapt.bf16(rng.standard_normal((B, Lq, Hq, D))) for _ in range(2))
    k, v = (adapt.bf16(rng.standard_normal((B, Lk, Hkv, D))) for _ in range(2))
    scale = D ** -0.5
    names = ("o", "gq", "gk", "gv")
    want = (adapt.attention(q, k, v, scale, causal)[0], *adapt.attention_backward(q, k, v, go, scale, causal))
    spread = adapt.attention_spread(q, k, v, scale, causal, None, go)

    def far(**how):
        return {name: adapt.off_in_norm(got, w, s) for name, got, w, s in zip(names, emulate(q, k, v, go, scale, causal, **how), want, spread)}

    assert all(f <= 1 for f in far().values()), far()
    for fault, wrong in FAULTS.items():
        f = far(operand_planes=1) if fault == "one plane" else far(fault=fault)
        assert all(f[name] > 1 for name in wrong), (fault, f)


def test_rounding_to_bf16():
    x = np.float32([1.0, 1 + 2.0 ** -8, 1 + 2.0 ** -8 + 2.0 ** -20, 1 + 3 * 2.0 ** -8, -3.14159, 0.0])
    assert adapt.bf16(x).tolist() == [1.0, 1.0, 1 + 2.0 ** -7, 1 + 2.0 ** -6, -3.140625, 0.0]
