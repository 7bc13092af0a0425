"""A transformer block's feed-forward part, trained with its activations kept in 8 bits, and its answers to single tokens.

    python examples/feed_forward.py [--tokens 4096] [--channels 320] [--hidden 1280] [--steps 100] [--keep blocks]

1. The output projection is frozen, its weights are 4-bit codes with a scale per 32 (fpq_block_quantize).
2. The norm's weights and both gated projections learn to give a teacher's output: norm on the residual stream, projections with the
   activation, output projection on its codes; backward the same in turn, AdamW on fp32 weights with the bf16 copies that the
   projections read.  What the backward pass needs is kept as 8-bit blocks (--keep blocks: the norm writes its result as them, the projections
   theirs) or as it is (--keep values).
3. Single tokens are answered by the same calls with one row.

Weights, tokens and the teacher are synthetic.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2408_06995_amd import binding as fpq  # noqa: E402

DEV = "cuda"
E2M1, EPS = (2, 1, 1, 6.0), 1e-6


def room(n):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=DEV)


def bytes_of(*shape):
    return torch.empty(shape, dtype=torch.uint8, device=DEV)


class FeedForward:
    """x [M, C] -> stream + W_out (a act(g)), with stream = x + residual and (a, g) = W norm(stream) + b."""

    def __init__(self, channels, hidden, dtype=torch.bfloat16, act=fpq.FPQ_GATE_SILU, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.C, self.N, self.dtype, self.act = channels, hidden, dtype, act
        self.type = fpq.FPQ_TYPE_BF16 if dtype == torch.bfloat16 else fpq.FPQ_TYPE_FP32
        self.norm = torch.ones(channels, device=DEV)
        self.w = torch.randn(2 * hidden, channels, generator=g, device=DEV) * channels ** -0.5
        self.w_read = self.w.to(dtype) if dtype != torch.float32 else self.w
        self.bias = torch.zeros(2 * hidden, device=DEV)
        out = torch.randn(channels, hidden, generator=g, device=DEV) * hidden ** -0.5
        self.codes, self.scales = bytes_of(channels, fpq.fpq_block_padded(hidden) // 2), bytes_of(channels, fpq.fpq_block_padded(hidden) // 32)
        fpq.fpq_block_quantize(out, E2M1, None, self.codes, self.scales)
        self.w_out = torch.empty(channels, hidden, dtype=dtype, device=DEV)        # their values, for the gradient of their input
        fpq.fpq_block_dequantize(self.codes, self.scales, E2M1, self.w_out)

    def workspaces(self, M):
        sizes = (fpq.fpq_gated_workspace_size(M, self.N, self.C, self.type), fpq.fpq_gated_backward_workspace_size(M, self.N, self.C, self.type),
                 fpq.fpq_block_linear_workspace_size(M, self.C, self.N, self.type), fpq.fpq_linear_backward_workspace_size(M, self.C, self.N, self.type),
                 fpq.fpq_rms_norm_backward_workspace_size(M, self.C))
        return room(max(sizes))                       # (one call after the other on one stream: they share it)

    def buffers(self, M, keep):
        """What a step writes, made once: results, what is kept for the backward pass, gradients."""
        t = dict(dtype=self.dtype, device=DEV)
        b = {"ws": self.workspaces(M), "stream": torch.empty(M, self.C, **t), "y": torch.empty(M, self.C, **t), "h": torch.empty(M, self.N, **t),
             "out": torch.empty(M, self.C, **t), "rstd": torch.empty(M, device=DEV), "x_scales": None, "pre": None, "pre_scales": None}
        if keep == "blocks":
            Cp, Np = fpq.fpq_block_padded(self.C), fpq.fpq_block_padded(self.N)
            b.update(x=bytes_of(M, Cp), x_scales=bytes_of(M, Cp // 32), pre=bytes_of(M, 2 * Np), pre_scales=bytes_of(M, 2 * Np // 32))
        elif keep == "values":
            b.update(x=b["y"], pre=torch.empty(M, 2 * self.N, **t))
        if keep:
            b.update(gh=torch.empty(M, self.N, **t), gy=torch.empty(M, self.C, **t), gx=torch.empty(M, self.C, **t), gw=torch.empty(2 * self.N, self.C, **t),
                     gb=torch.empty(2 * self.N, device=DEV), gnorm=torch.empty(self.C, device=DEV))
        return b

    def forward(self, x, residual, b):
        kept = (b["x"], None, None, None, b["x_scales"]) if b["x_scales"] is not None else ()
        fpq.fpq_rms_norm(x, residual, self.norm, EPS, b["stream"], b["y"], b["rstd"], *kept)
        fpq.fpq_gated(b["y"], self.w_read, self.bias, self.act, b["h"], b["pre"], b["pre_scales"], b["ws"])
        fpq.fpq_block_linear(b["h"], self.codes, self.scales, None, b["out"], b["ws"])
        return b["out"]                               # (the stream goes on beside it)

    def backward(self, g_out, g_stream, b):
        """Gradients of norm, w, bias and of the stream's inputs for those of `out` and of the stream behind this block."""
        fpq.fpq_linear_backward(None, None, self.w_out, g_out, b["gh"], None, None, b["ws"])
        fpq.fpq_gated_backward(b["x"], b["x_scales"], self.w_read, b["pre"], b["pre_scales"], self.act, b["gh"], b["gy"], b["gw"], b["gb"], b["ws"])
        fpq.fpq_rms_norm_backward(b["stream"], self.norm, b["rstd"], b["gy"], g_stream, b["gx"], b["gnorm"], b["ws"])
        return b["gx"]


def adamw(block, b):
    """A plan for the block's weights: (step number, learning rate) -> a step."""
    items = []
    for p, grad, copy in ((block.w, b["gw"], block.w_read if block.w_read is not block.w else None), (block.bias, b["gb"], None), (block.norm, b["gnorm"], None)):
        items.append((p.view(-1), grad.view(-1), torch.zeros(p.numel(), device=DEV), torch.zeros(p.numel(), device=DEV), None, None,
                      None if copy is None else copy.view(-1)))
    tensors = fpq.adamw_tensors(items)
    plan = room(fpq.fpq_adamw_plan_size(tensors))
    pieces = fpq.fpq_adamw_plan(tensors, plan)

    def step(i, lr, keep=items):
        fpq.fpq_adamw_step(plan, pieces, lr, 0.9, 0.999, 1e-8, 0.0, i)
    return step


def train(block, teacher, x, residual, steps, keep, lr=2e-3):
    M = x.shape[0]
    b = block.buffers(M, keep)
    target = teacher.forward(x, residual, teacher.buffers(M, None)).float()
    step, losses = adamw(block, b), []
    for i in range(steps):
        error = block.forward(x, residual, b).float() - target
        losses.append(error.square().mean())
        block.backward((error * (2.0 / error.numel())).to(block.dtype), None, b)
        step(i + 1, lr)
    return torch.stack(losses).tolist()


def run(tokens=4096, channels=320, hidden=1280, steps=100, keep="blocks", dtype=torch.bfloat16, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x, residual = (torch.randn(tokens, channels, generator=g, device=DEV).to(dtype) for _ in range(2))
    block, teacher = FeedForward(channels, hidden, dtype, seed=1), FeedForward(channels, hidden, dtype, seed=1)
    block.w.copy_(torch.randn(block.w.shape, generator=g, device=DEV) * channels ** -0.5)
    block.w_read.copy_(block.w)
    losses = train(block, teacher, x, residual, steps, keep)
    # a token of each of four requests
    answer = block.forward(x[:4], residual[:4], block.buffers(4, None)).clone()
    return losses, answer, (block, x, residual)


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("tokens", 4096), ("channels", 320), ("hidden", 1280), ("steps", 100)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--keep", choices=["blocks", "values"], default="blocks")
    losses, answer, _ = run(**vars(ap.parse_args()))
    for i in sorted({*range(0, len(losses), 20), len(losses) - 1}):
        print("step %3d  squared error of the output %.3e" % (i, losses[i]))
    print("answers to a token of each of four requests:", tuple(answer.shape))


if __name__ == "__main__":
    main()
