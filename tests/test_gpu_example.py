"""The example of adapters at a quantized attention layer, at a small size: it learns, and what it serves is what the formulas give."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("adapt_attention", os.path.join(ROOT, "examples", "adapt_attention.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.fixture(scope="module")
def done():
    return example(), example().run(images=3, tokens=100, channels=64, heads=4, rank=8, steps=120, rounding_steps=40)


def test_learns(done):
    _, (errors, losses, _, _) = done
    assert errors[1] < errors[0]                     # learned rounding is better than rounding to nearest
    assert losses[-1] < 0.5 * losses[0] and all(b < 2 * losses[0] for b in losses)


def test_answers(done):
    """Each answer against the same row of plain attention in 64 bits on the projection that the layer gave."""
    ex, (_, _, answer, (layer, x, _, of, lens)) = done
    B, L, C = x.shape
    assert answer.shape == (B, 1, layer.heads, C // layer.heads)
    plain = torch.empty(B * L, 3 * C, device=x.device)
    rows = x.reshape(B * L, C)
    layer.projection(rows, plain, layer.projection.workspace(B * L))
    token = x[:, 0].contiguous()
    plain_q = torch.empty(B, 3 * C, device=x.device)
    layer.projection(token, plain_q, layer.projection.workspace(B))
    plain, plain_q = plain.view(B, L, 3 * C).double().cpu(), plain_q.double().cpu()
    a, b, x, token = layer.a.double().cpu(), layer.b.double().cpu(), x.double().cpu(), token.double().cpu()
    for i, adapter in enumerate(of[:-1] + [-1]):
        y, q = plain[i], plain_q[i]
        if adapter >= 0:
            y, q = y + x[i] @ a[adapter].T @ b[adapter].T, q + token[i] @ a[adapter].T @ b[adapter].T
        y, q = y.view(L, 3, layer.heads, -1)[: lens[i]], q.view(3, layer.heads, -1)[0]
        s = torch.einsum("hd,lhd->hl", q, y[:, 1]) * layer.scale
        want = torch.einsum("hl,lhd->hd", torch.softmax(s, 1), y[:, 2])
        # sums of fp32 products over C, rank and L terms of magnitude 1, each 2^-24 of its partial sums, and the exponential of scores
        # that carry such errors: 2^-24 (C + rank + L) at most, of values of at most 8
        assert (answer[i, 0].double().cpu() - want).abs().max() < 8 * 2.0 ** -24 * (C + layer.rank + L) * 2
