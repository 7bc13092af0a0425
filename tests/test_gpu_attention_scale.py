"""Attention at the smallest and largest scale that is accepted."""
import pytest
import torch

from test_gpu_attention import both, tensors

pytestmark = pytest.mark.gpu

#: few rows (keys form), few rows on parts of the keys, many rows, rows on two parts
SHAPES = [(2, 3, 40, 4, 2, 64), (1, 2, 3000, 2, 1, 32), (3, 300, 300, 8, 8, 40), (2, 1000, 600, 2, 2, 80)]


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("shape", SHAPES)
def test_ends_of_the_scale(shape, causal, t):
    print(shape, causal, t, flush=True)
    q, k, v, go = tensors(*shape, t, 91)
    # scores of ordinary size, from operands that make up for the scale
    both(q * 2.0 ** 49, k * 2.0 ** 48, v, go, causal, None, scale=2.0 ** -100)
    both(q * 2.0 ** -52, k * 2.0 ** -51, v, go, causal, None, scale=2.0 ** 100)
    # no scores to speak of: averages
    both(q, k, v, go, causal, None, scale=2.0 ** -100)
    both(torch.zeros_like(q), k, v, go, causal, None, scale=2.0 ** 100)
