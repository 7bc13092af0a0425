"""The oracle of the operators for adapting a model, checked by itself: gradients against differences."""
import numpy as np
import pytest

from oracle import adapt


@pytest.mark.parametrize("causal,lens,heads", [(False, None, 2), (True, None, 4), (True, [5, 0, 2], 2), (False, [7, 1, 0], 4)])
def test_attention_gradient_against_differences(causal, lens, heads):
    rng = np.random.default_rng(3)
    q, go = (rng.standard_normal((3, 6, heads, 5)) for _ in range(2))
    k, v = (rng.standard_normal((3, 7, 2, 5)) for _ in range(2))
    loss = lambda q, k, v: (adapt.attention(q, k, v, 0.7, causal, lens)[0] * go).sum()
    for x, g in zip((0, 1, 2), adapt.attention_backward(q, k, v, go, 0.7, causal, lens)):
        args = [q, k, v]
        step = rng.standard_normal(args[x].shape)
        h = 1e-5
        up, down = ([a + s * h * step if n == x else a for n, a in enumerate(args)] for s in (1, -1))
        difference = (loss(*up) - loss(*down)) / (2 * h)
        assert abs(difference - (g * step).sum()) <= 1e-8 * np.abs(g * step).sum() + 1e-9


def test_attention_of_rows_that_see_nothing():
    rng = np.random.default_rng(4)
    q, k, v = rng.standard_normal((2, 5, 1, 4)), rng.standard_normal((2, 3, 1, 4)), rng.standard_normal((2, 3, 1, 4))
    o, lse = adapt.attention(q, k, v, 1.0, True, [3, 0])
    assert np.all(o[0, :2] == 0) and np.all(np.isneginf(lse[0, 0, :2])) and np.all(o[1] == 0) and np.all(np.isneginf(lse[1]))
    assert np.allclose(o[0, 2], v[0, 0]) and np.isclose(lse[0, 0, 2], (q[0, 2] * k[0, 0]).sum())


def test_state_codes_are_the_nearest():
    values = adapt.e4m3_values()
    assert values[126] == 448 and values[8] == 2.0 ** -6 and values[1] == 2.0 ** -9 and values[254] == -448
    finite = values[np.isfinite(values)]
    assert np.array_equal(adapt.e4m3_codes(finite), np.arange(256)[np.isfinite(values)])
    x = np.random.default_rng(5).standard_normal(4000).astype(np.float32) * np.float32(100)
    x = np.clip(x, -448, 448)
    got = values[adapt.e4m3_codes(x)]
    assert np.all(np.abs(got - x) <= np.abs(finite[:, None] - x).min(0))
    assert adapt.e4m3_codes(np.float32([1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10]))[:4].tolist() == [56, 58, 0, 2]


def test_adamw_step_is_the_textbook_one():
    rng = np.random.default_rng(6)
    p, g, m = (rng.standard_normal(50) for _ in range(3))
    v = rng.random(50)
    new, m1, v1 = adapt.adamw(p, g, m, v, 0.01, 0.9, 0.99, 1e-6, 0.1, 7, 0.5)
    m2, v2 = 0.9 * m + 0.1 * (g / 2), 0.99 * v + 0.01 * (g / 2) ** 2
    want = p - 0.01 * (0.1 * p + (m2 / (1 - 0.9 ** 7)) / (np.sqrt(v2 / (1 - 0.99 ** 7)) + 1e-6))
    assert np.allclose(m1, m2) and np.allclose(v1, v2) and np.allclose(new, want, rtol=1e-12)


def test_adapter_gradient_against_differences():
    rng = np.random.default_rng(8)
    starts, of = [1, 4, 4, 9, 11], [2, 0, 0, -1]
    x, base, gy = rng.standard_normal((12, 6)), rng.standard_normal((12, 5)), rng.standard_normal((12, 5))
    a, b, s = rng.standard_normal((3, 2, 6)), rng.standard_normal((3, 5, 2)), np.array([0.5, 2.0, 1.5])
    loss = lambda x, a, b: (adapt.adapter_apply(x, a, b, s, starts, of, base)[0] * gy).sum()
    grads = adapt.adapter_backward(x, a, b, s, starts, of, gy, np.zeros_like(x))
    for k, g in enumerate(grads):
        args = [x, a, b]
        step, h = rng.standard_normal(args[k].shape), 1e-5
        up, down = ([v + z * h * step if n == k else v for n, v in enumerate(args)] for z in (1, -1))
        assert abs((loss(*up) - loss(*down)) / (2 * h) - (g * step).sum()) <= 1e-8 * np.abs(g * step).sum() + 1e-9
    y, t = adapt.adapter_apply(x, a, b, s, starts, of, base)
    assert np.array_equal(y[[0, 9, 10, 11]], base[[0, 9, 10, 11]]) and np.all(t[9:] == 0) and np.all(grads[1][1] == 0)
