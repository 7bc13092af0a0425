"""SiLU's gradient where the gate is far below zero: the slope is of the sigmoid's size there, and so is its bound."""
import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2408_06995_amd import binding as B

GATES = np.concatenate([np.linspace(-80, -8, 289), np.linspace(-8, 80, 177)])


def test_the_bound_is_of_the_slopes_size():
    """A slope of zero, of the wrong sign or a percent off is outside it."""
    g = GATES[GATES <= -8]
    _, slope, _, off = blocks.gate(g, "silu")
    assert (slope < 0).all() and (off < 0.01 * np.abs(slope)).all()
    # the formula in fp32, one rounding after the other
    f = np.float32
    x = GATES.astype(f)
    z = f(1) / (f(1) + np.exp(-x))
    got = z * (f(1) + x * (f(1) - z))
    _, slope, _, off = blocks.gate(GATES, "silu")
    assert (np.abs(got - slope) <= off).all()


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_gradient_of_the_gates(t):
    """One row's dg itself: the bias's gradient, which is not rounded to the type."""
    from gpu_util import DEV
    from test_gpu_blocks import TYPES, host, nan, room
    N = len(GATES)
    g = torch.from_numpy(GATES).to(TYPES[t])
    pre = torch.cat([torch.linspace(0.5, 2, N).to(TYPES[t]), g]).view(1, -1).to(DEV)
    gh = torch.linspace(1, 3, N).to(TYPES[t]).view(1, -1).to(DEV)
    x, w, gb = torch.ones(1, 8, dtype=TYPES[t], device=DEV), torch.ones(2 * N, 8, dtype=TYPES[t], device=DEV), nan(2 * N)
    B.fpq_gated_backward(x, None, w, pre, None, B.FPQ_GATE_SILU, gh, None, None, gb, room(B.fpq_gated_backward_workspace_size(1, N, 8, int(t == "bf16"))))
    want, off = blocks.gated_backward(host(x), host(w), host(pre[:, :N]), host(pre[:, N:]), "silu", host(gh), t == "bf16")[2]
    got = host(gb)
    assert (np.abs(got - want) <= off).all(), np.max(np.abs(got - want) / off)
    assert (off[N:][:289] <= 0.01 * np.abs(want[N:][:289])).all()
