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
