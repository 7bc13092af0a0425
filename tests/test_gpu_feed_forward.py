"""The operators around a block's projections as they are used together, in the example of a feed-forward block: its gradients against the
formulas', a training step captured in a graph, two steps side by side on two streams."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2408_06995_amd import binding as B
from gpu_util import DEV
from test_gpu_blocks import host

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U32 = 2.0 ** -24


def example():
    spec = importlib.util.spec_from_file_location("feed_forward", os.path.join(ROOT, "examples", "feed_forward.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def inputs(M, C, dtype, seed=3):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(M, C, generator=g).to(dtype).to(DEV) for _ in range(4)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,C,N", [(3, 64, 96), (40, 72, 130), (200, 128, 320)])
def test_gradients_of_the_whole_block(M, C, N, act):
    """fp32, values kept: the chain of all five calls against the formulas in 64 bits.  Every product of the chain makes an error of its sum's length, and the
    activation one of up to 2 (4 + |g|) 2^-23 or 6e-7, times what it multiplies: in all (M + 2 N + 2 C + 64) 2^-24 of the chain of magnitudes."""
    ex = example()
    block = ex.FeedForward(C, N, torch.float32, B.FPQ_GATE_SILU if act == "silu" else B.FPQ_GATE_GELU, seed=2)
    block.norm.copy_(torch.linspace(0.5, 1.5, C))
    block.bias.copy_(torch.linspace(-0.5, 0.5, 2 * N))
    x, residual, g_out, g_stream = inputs(M, C, torch.float32)
    b = block.buffers(M, "values")
    out = block.forward(x, residual, b).clone()
    gx = block.backward(g_out, g_stream, b)
    w, bias, norm, w_out = host(block.w), host(block.bias), host(block.norm), host(block.w_out)
    r = host(x + residual)
    y, _, rstd, _ = blocks.rms_norm(r, norm, ex.EPS)
    h, _, (a, g), _ = blocks.gated(y, w, bias, act, False)
    gh = host(g_out) @ w_out
    (gy, _), (gw, _), (gb, _) = blocks.gated_backward(y, w, a, g, act, gh, False)
    want_x, _, gnorm, _ = blocks.rms_norm_backward(r, norm, rstd, gy, host(g_stream))
    # magnitudes
    f, slope, _, _ = blocks.gate(g, act)
    A = lambda v: np.abs(v)
    m_pre = A(y) @ A(w).T + A(bias)
    m_a, m_g = m_pre[:, :N], m_pre[:, N:]
    m_h = m_a * (A(f) + 1.13 * m_g)
    m_gh = A(host(g_out)) @ A(w_out)
    m_d = np.concatenate([m_gh * (A(f) + 1.13 * m_g), m_gh * (m_a * (1.13 + m_g))], 1)
    m_gy = m_d @ A(w)
    m_x = rstd[:, None] * (m_gy * norm + A(r) * (m_gy * norm * A(r)).mean(1, keepdims=True) * rstd[:, None] ** 2) + A(host(g_stream))
    rel = (M + 2 * N + 2 * C + 64) * U32
    for name, got, ref, mass in (("out", out, h @ w_out.T, m_h @ A(w_out).T), ("gw", b["gw"], gw, m_d.T @ A(y)), ("gb", b["gb"], gb, m_d.sum(0)),
                                 ("gx", gx, want_x, m_x), ("gnorm", b["gnorm"], gnorm, (m_gy * A(r) * rstd[:, None]).sum(0))):
        err = np.abs(host(got) - ref)
        assert (err <= rel * mass + 1e-30).all(), "%s: worst %.3g of the bound" % (name, (err / (rel * mass + 1e-30)).max())


@pytest.mark.parametrize("keep", ["blocks", "values"])
def test_gradients_from_what_is_kept(keep):
    """bf16: each gradient is the formulas' from what the step kept of the forward pass, within the bounds of its own call."""
    ex = example()
    M, C, N = 150, 96, 160
    block = ex.FeedForward(C, N, seed=4)
    x, residual, g_out, g_stream = inputs(M, C, torch.bfloat16)
    b = block.buffers(M, keep)
    block.forward(x, residual, b)
    gx = block.backward(g_out, g_stream, b)
    if keep == "blocks":
        xv = blocks.block_values(b["x"].cpu().numpy(), b["x_scales"].cpu().numpy(), 8, C)
        c, s = b["pre"].cpu().numpy(), b["pre_scales"].cpu().numpy()
        a, g = (blocks.block_values(c[:, i * N:(i + 1) * N], s[:, i * N // 32:(i + 1) * N // 32], 8, N) for i in range(2))
        # the norm's blocks are its result to half a step of their codes
        y = blocks.rms_norm(host(b["stream"]), np.ones(C), ex.EPS)[0]
        unit = np.repeat(2.0 ** (b["x_scales"].cpu().numpy().astype(float) - 127), 32, 1)[:, :C]
        assert (np.abs(xv - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * unit) * (1 + 2.0 ** -10)).all()
    else:
        xv, a, g = host(b["y"]), host(b["pre"][:, :N]), host(b["pre"][:, N:])
    (wy, oy), (ww, ow), (wb, ob) = blocks.gated_backward(xv, host(block.w_read), a, g, "silu", host(b["gh"]), True)
    for name, got, want, off in (("gy", b["gy"], wy, oy), ("gw", b["gw"], ww, ow), ("gb", b["gb"], wb, ob)):
        assert (np.abs(host(got) - want) <= off).all(), name
    wx, ox, wn, on = blocks.rms_norm_backward(host(b["stream"]), np.ones(C), host(b["rstd"]), host(b["gy"]), host(g_stream))
    assert (np.abs(host(gx) - wx) <= ox + 2.0 ** -8 * (np.abs(wx) + ox)).all() and (np.abs(host(b["gnorm"]) - wn) <= on).all()


@pytest.mark.parametrize("keep", ["blocks", "values"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("M", [2, 40, 300])
def test_captured_step(M, dtype, keep):
    """Forward, backward and AdamW in a graph: every replay, with other inputs and eager work between, gives the eager step's bits."""
    ex = example()
    C, N = 72, 200

    def fresh():
        block = ex.FeedForward(C, N, dtype, seed=5)
        b = block.buffers(M, keep)
        return block, b, ex.adamw(block, b)

    feeds = [inputs(M, C, dtype, seed=10 + i) for i in range(5)]

    def step(block, b, opt, data):
        block.forward(data[0], data[1], b)
        block.backward(data[2], data[3], b)
        opt(1, 1e-2)

    eager, eb, eo = fresh()
    want = []
    for f in feeds:
        step(eager, eb, eo, f)
        torch.cuda.synchronize()
        want.append([t.clone() for t in (eb["out"], eb["gx"], eb["gw"], eb["gnorm"], eager.w, eager.norm)])
    block, b, opt = fresh()
    data = [torch.empty_like(t) for t in feeds[0]]
    side = torch.cuda.Stream()
    warm, wb, wo = fresh()
    with torch.cuda.stream(side):
        step(warm, wb, wo, feeds[0])
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(block, b, opt, data)
    torch.cuda.synchronize()
    for f, w in zip(feeds, want):
        for t, v in zip(data, f):
            t.copy_(v)
        other = torch.randn(1 << 16, device=DEV).sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip((b["out"], b["gx"], b["gw"], b["gnorm"], block.w, block.norm), w):
            assert torch.equal(got, ref)
        assert torch.isfinite(other)


def test_two_streams():
    """Two blocks' steps at once, with workspaces of their own."""
    ex = example()
    sizes = ((300, 128, 320), (90, 72, 130))
    made = []
    for i, (M, C, N) in enumerate(sizes):
        block = ex.FeedForward(C, N, seed=6 + i)
        made.append((block, inputs(M, C, torch.bfloat16, 20 + i), block.buffers(M, "blocks"), block.buffers(M, "blocks")))

    def step(block, data, b):
        block.forward(data[0], data[1], b)
        block.backward(data[2], data[3], b)

    for block, data, b, _ in made:
        step(block, data, b)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(5):
        for s, (block, data, _, b) in zip(streams, made):
            with torch.cuda.stream(s):
                step(block, data, b)
    torch.cuda.synchronize()
    for _, _, b, c in made:
        for k in ("out", "gx", "gw", "gb", "gnorm", "pre", "x"):
            assert torch.equal(b[k], c[k]), k


@pytest.mark.parametrize("keep", ["blocks", "values"])
def test_example_runs(keep):
    ex = example()
    losses, answer, (block, x, residual) = ex.run(tokens=200, channels=64, hidden=96, steps=30, keep=keep)
    assert len(losses) == 30 and all(np.isfinite(losses)) and answer.shape == (4, 64)
    # the answers are what the formulas give for the weights that were learned
    y, oy = blocks.rms_norm(host((x[:4].float() + residual[:4].float()).bfloat16()), host(block.norm), ex.EPS)[:2]
    b = block.buffers(4, None)
    block.forward(x[:4], residual[:4], b)
    assert torch.equal(b["out"], answer)
    assert (np.abs(host(b["y"]) - y) <= oy + 2.0 ** -8 * (np.abs(y) + oy)).all()
    h, oh, _, _ = blocks.gated(host(b["y"]), host(block.w_read), host(block.bias), "silu", True)
    assert (np.abs(host(b["h"]) - h) <= oh).all()
    out, oo = blocks.block_linear(host(b["h"]), host(block.w_out), None, True)
    assert (np.abs(host(answer) - out) <= oo).all()
