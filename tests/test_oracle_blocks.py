"""The oracle of the operators around the projections against what it must give: nearest values by search, gradients by differences."""
import numpy as np
import pytest

from oracle import blocks


@pytest.mark.parametrize("bits", [8, 4])
def test_codes_are_nearest(bits):
    rng = np.random.default_rng(bits)
    x = rng.standard_normal((7, 70)) * np.exp(rng.standard_normal((7, 1)) * 5)
    x[0, :32] = 0
    codes, scales = blocks.block_quantize(x, bits)
    v = blocks.block_values(codes, scales, bits, 70)
    grid = blocks.e4m3_values() if bits == 8 else blocks.E2M1
    s = 2.0 ** (scales.astype(float) - 127)
    top = np.abs(blocks._in_blocks(x)).max(2)
    assert np.all(top <= grid[-1] * s) and np.all((top > grid[-1] * s / 2) | (top == 0)) and np.all(s[top == 0] == 1)
    for m in range(7):
        for k in range(70):
            near = np.abs(np.concatenate([grid, -grid]) * s[m, k // 32] - x[m, k]).min()
            assert abs(v[m, k] - x[m, k]) == near
    # a tie goes to the even one
    tie = np.zeros((1, 32))
    tie[0, :3] = [grid[-1], (grid[3] + grid[4]) / 2, (grid[4] + grid[5]) / 2]
    assert (blocks.block_quantize(tie, bits)[0][0, 1:3] & (127 if bits == 8 else 7)).tolist() == [4, 4]


def test_mask_rounds_up_or_down():
    rng = np.random.default_rng(3)
    w, mask = rng.standard_normal((4, 64)), rng.integers(0, 2, (4, 64))
    codes, scales = blocks.block_quantize(w, 4, mask)
    v, s = blocks.block_values(codes, scales, 4, 64), np.repeat(2.0 ** (scales.astype(float) - 127), 32, 1)
    assert np.all(np.where(mask == 1, v - w > -1e-12, v - w < 1e-12))
    assert np.all(np.abs(v - w) <= 2 * s)
    assert blocks.unpack(blocks.nibbles(codes)).tolist() == codes.tolist()


def test_infinities_make_a_block_nan():
    x = np.ones((2, 64))
    x[0, 5], x[1, 40] = np.inf, np.nan
    codes, scales = blocks.block_quantize(x, 8)
    v = blocks.block_values(codes, scales, 8, 64)
    assert np.isnan(v[0, :32]).all() and np.isnan(v[1, 32:]).all() and np.isfinite(v[0, 32:]).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_gradients_by_differences(act):
    rng = np.random.default_rng(5)
    x, w, b, gh = rng.standard_normal((3, 6)), rng.standard_normal((10, 6)), rng.standard_normal(10), rng.standard_normal((3, 5))
    loss = lambda x, w, b: (blocks.gated(x, w, b, act, False)[0] * gh).sum()
    a, g = blocks.gated(x, w, b, act, False)[2]
    (gx, _), (gw, _), (gb, _) = blocks.gated_backward(x, w, a, g, act, gh, False)
    for at, grad, call in ((x, gx, lambda v: loss(v, w, b)), (w, gw, lambda v: loss(x, v, b)), (b, gb, lambda v: loss(x, w, v))):
        for i in np.ndindex(at.shape):
            d = np.zeros(at.shape)
            d[i] = 1e-5
            assert abs((call(at + d) - call(at - d)) / 2e-5 - grad[i]) < 1e-7


def test_norm_gradients_by_differences():
    rng = np.random.default_rng(7)
    r, w, gy, gs = rng.standard_normal((3, 9)), rng.standard_normal(9), rng.standard_normal((3, 9)), rng.standard_normal((3, 9))
    loss = lambda r, w: (blocks.rms_norm(r, w, 0.1)[0] * gy).sum() + (r * gs).sum()
    gx, _, gw, _ = blocks.rms_norm_backward(r, w, blocks.rms_norm(r, w, 0.1)[2], gy, gs)
    for at, grad, call in ((r, gx, lambda v: loss(v, w)), (w, gw, lambda v: loss(r, v))):
        for i in np.ndindex(at.shape):
            d = np.zeros(at.shape)
            d[i] = 1e-5
            assert abs((call(at + d) - call(at - d)) / 2e-5 - grad[i]) < 1e-7


def test_linear_gradients():
    rng = np.random.default_rng(9)
    x, w, gy = rng.standard_normal((4, 5)), rng.standard_normal((3, 5)), rng.standard_normal((4, 3))
    (gx, _), (gw, _), (gb, _) = blocks.linear_backward(x, w, gy, False)
    for i in np.ndindex(x.shape):
        d = np.zeros(x.shape)
        d[i] = 1.0
        assert abs(((x + d) @ w.T * gy).sum() - (x @ w.T * gy).sum() - gx[i]) < 1e-12
    assert np.allclose(gw, sum(np.outer(gy[m], x[m]) for m in range(4))) and np.allclose(gb, gy.sum(0))
