"""Adapters of an attention layer whose projection is quantized, from rounding to serving.

    python examples/adapt_attention.py [--images 4] [--tokens 1024] [--channels 320] [--heads 8] [--rank 16] [--steps 100]

1. The query / key / value projection is quantized to FP4, its rounding learned by AdamW with 8-bit states on the gradient of
   fpq_rl_step.
2. Two tasks have a teacher each: the same layer in full precision, with weights a little different.  A low-rank adapter per task
   learns to give its teacher's attention output: projection on codes + adapters, attention, its gradient, the adapters' gradient,
   AdamW; images of both tasks are in one batch.
3. Requests of both tasks, and one without an adapter, are answered together: a new token each, which reads its image's keys.

Weights, images and teachers are synthetic.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2408_06995_amd import binding as fpq, synth  # noqa: E402

DEV = "cuda"


def room(n):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=DEV)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class AdamW:
    """Steps for a list of tensors: one plan, one launch a step."""

    def __init__(self, params, grads, lr, eight_bits=False, copies=None):
        self.lr, self.steps, self.state = lr, 0, []
        for p, g, c in zip(params, grads, copies or [None] * len(params)):
            n = p.numel()
            if eight_bits:
                m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in "mv")
                scales = [torch.ones((n + 255) // 256, device=DEV) for _ in "mv"]
            else:
                m, v = (torch.zeros(n, device=DEV) for _ in "mv")
                scales = [None, None]
            self.state.append((p, g, m, v, *scales, c))
        tensors = fpq.adamw_tensors(self.state)
        self.plan = room(fpq.fpq_adamw_plan_size(tensors))
        self.pieces = fpq.fpq_adamw_plan(tensors, self.plan)

    def step(self):
        self.steps += 1
        fpq.fpq_adamw_step(self.plan, self.pieces, self.lr, 0.9, 0.999, 1e-8, 0.0, self.steps)


class Projection:
    """[M, K] fp32 -> [M, N] fp32 on E2M1 weights and E4M3 activations (scale found in the call)."""

    def __init__(self, w, mask=None):
        self.N, self.K = w.shape
        self.packed = room(fpq.fpq_packed_size(self.N, self.K, 1, 1, synth.E2M1))
        self.scale = torch.empty(self.N, device=DEV)
        fpq.fpq_pack_weights(w, synth.E2M1, None, mask, self.packed, self.scale, None)

    def __call__(self, x, y, workspace):
        fpq.fpq_gemm(x, fpq.FPQ_X_FP32_DYNAMIC, synth.E4M3, 0.0, None, self.packed, synth.E2M1, self.scale, None, y, x.shape[0], self.N,
                     self.K, fpq.FPQ_ACC_FP32, workspace)

    def workspace(self, M):
        return room(fpq.fpq_gemm_workspace_size(M, self.N, self.K, fpq.FPQ_X_FP32_DYNAMIC))


def learn_rounding(w, x, steps, lr=0.05):
    """The mask of rounding learning on the rows x."""
    nearest = Projection(w)
    N, K = w.shape
    alpha, grad, loss = torch.empty_like(w), torch.empty_like(w), torch.empty(2, device=DEV)
    fpq.fpq_rl_init_alpha(w, nearest.scale, synth.E2M1, alpha)
    ws = room(fpq.fpq_rl_workspace_size(x.shape[0], N, K))
    optimizer = AdamW([alpha], [grad], lr, eight_bits=True)
    for i in range(steps):
        # (its own descent step has the rate zero: AdamW makes it)
        fpq.fpq_rl_step(w, nearest.scale, synth.E2M1, alpha, x, 0.0, 10.0 * i / steps, loss, grad, ws)
        optimizer.step()
    mask = torch.empty(N, K, dtype=torch.uint8, device=DEV)
    fpq.fpq_rl_mask(alpha, mask)
    return mask


class Layer:
    """Attention of quantized q, k and v, with a pool of adapters at the projection."""

    def __init__(self, projection, heads, adapters, rank, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.projection, self.heads, self.rank = projection, heads, rank
        self.C = projection.K
        self.scale = (self.C // heads) ** -0.5
        self.a = torch.randn(adapters, rank, self.C, generator=g, device=DEV) * self.C ** -0.5
        self.b = torch.zeros(adapters, 3 * self.C, rank, device=DEV)
        self.scaling = torch.ones(adapters, device=DEV)

    def sizes(self, M, requests):
        return M, 3 * self.C, self.C, self.rank, requests, self.a.shape[0]

    def project(self, x, starts, of, t=None):
        """x [M, C] -> [M, 3, heads, C / heads]: on codes, and each request's adapter on top, in place."""
        M = x.shape[0]
        y = torch.empty(M, 3 * self.C, device=DEV)
        self.projection(x, y, self.projection.workspace(M))
        fpq.fpq_adapter_apply(x, self.a, self.b, self.scaling, starts, of, y, y, t, room(fpq.fpq_adapter_workspace_size(*self.sizes(M, len(of)))))
        return y.view(M, 3, self.heads, -1)

    def attend(self, q, k, v, lse=None, lens=None):
        o = torch.empty(q.shape, device=DEV)
        size = fpq.fpq_attention_workspace_size(q.shape[0], self.heads, self.heads, q.shape[1], k.shape[1], q.shape[3], fpq.FPQ_TYPE_FP32)
        fpq.fpq_attention(q, k, v, o, lse, self.scale, 0, lens, room(size))
        return o


def split(y, B):
    """q, k and v of B images as columns of the projection's result: strided views, nothing is copied."""
    return [y.view(B, -1, *y.shape[1:])[:, :, i] for i in range(3)]


def train(layer, x, target, of, steps, lr=2e-3):
    """x [B, tokens, C], target [B, tokens, heads, C / heads]; image i has the adapter of[i].  Returns the losses."""
    B, L, C = x.shape
    D = C // layer.heads
    rows, starts = x.reshape(B * L, C), ints([i * L for i in range(B + 1)])
    ga, gb = torch.empty_like(layer.a), torch.empty_like(layer.b)
    optimizer = AdamW([layer.a, layer.b], [ga, gb], lr)
    t, lse = torch.empty(B * L, layer.rank, device=DEV), torch.empty(B, layer.heads, L, device=DEV)
    gy = torch.empty(B * L, 3, layer.heads, D, device=DEV)
    ws = room(fpq.fpq_attention_backward_workspace_size(B, layer.heads, layer.heads, L, L, D, fpq.FPQ_TYPE_FP32))
    ws_adapter = room(fpq.fpq_adapter_backward_workspace_size(*layer.sizes(B * L, B)))
    losses = []
    for _ in range(steps):
        q, k, v = split(layer.project(rows, starts, of, t), B)
        o = layer.attend(q, k, v, lse)
        error = o - target
        losses.append((error * error).mean())
        go = error * (2.0 / error.numel())
        fpq.fpq_attention_backward(q, k, v, o, lse, go, *split(gy, B), layer.scale, 0, None, ws)
        # the codes' weights stay as they are, and nothing ahead of the layer learns: no gradient of x
        fpq.fpq_adapter_backward(rows, layer.a, layer.b, layer.scaling, starts, of, t, gy.view(B * L, 3 * C), None, None, ga, gb, ws_adapter)
        optimizer.step()
    return torch.stack(losses).tolist()


def serve(layer, x, lens, of, token):
    """The answers to token [B, C], one row of each image's request: attention over the first lens[i] tokens of image x[i]."""
    B, L, C = x.shape
    _, k, v = split(layer.project(x.reshape(B * L, C), ints([i * L for i in range(B + 1)]), of), B)
    q, _, _ = split(layer.project(token, ints(list(range(B + 1))), of), B)
    return layer.attend(q, k, v, None, lens)


def teacher(w, delta, x, heads):
    """Attention of the full-precision layer in plain torch: the targets."""
    B, L, C = x.shape
    q, k, v = ((x @ (w + delta).t()).view(B, L, 3, heads, C // heads).permute(2, 0, 3, 1, 4).contiguous())
    return (torch.softmax((q @ k.transpose(2, 3).contiguous()) * (C // heads) ** -0.5, 3) @ v).permute(0, 2, 1, 3).contiguous()


def run(images=4, tokens=1024, channels=320, heads=8, rank=16, steps=100, rounding_steps=200, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV)
    w = randn(3 * channels, channels) * channels ** -0.5
    # (channels that go together, as activations do: rounding to nearest is best for independent ones)
    spectrum = 3.0 / (1.0 + 16.0 * torch.arange(channels, device=DEV) / channels)
    x = (randn(images, tokens, channels) * spectrum) @ torch.linalg.qr(randn(channels, channels))[0]
    mask = learn_rounding(w, x.view(-1, channels)[:2048].contiguous(), rounding_steps)

    def output_error(p):
        rows = x.view(-1, channels)
        y = torch.empty(rows.shape[0], 3 * channels, device=DEV)
        p(rows, y, p.workspace(rows.shape[0]))
        return (y - rows @ w.t()).square().mean().item()

    learned = Projection(w, mask)
    errors = output_error(Projection(w)), output_error(learned)

    tasks = [(randn(3 * channels, 4) @ randn(4, channels)) * (0.3 * channels ** -0.5) for _ in range(2)]
    of = [i % 2 for i in range(images)]
    target = torch.cat([teacher(w, tasks[of[i]], x[i:i + 1], heads) for i in range(images)])
    layer = Layer(learned, heads, 2, rank, seed)
    losses = train(layer, x, target, ints(of), steps)

    # the last image's request has no adapter, and lengths differ
    lens = [tokens - 7 * i for i in range(images)]
    answer = serve(layer, x, ints(lens), ints(of[:-1] + [-1]), x[:, 0].contiguous())
    return errors, losses, answer, (layer, x, target, of, lens)


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("images", 4), ("tokens", 1024), ("channels", 320), ("heads", 8), ("rank", 16), ("steps", 100), ("rounding-steps", 200)):
        ap.add_argument("--" + name, type=int, default=value)
    errors, losses, answer, _ = run(**vars(ap.parse_args()))
    print("projection, squared error of its output: rounded to nearest %.3e, rounding learned %.3e" % errors)
    for i in sorted({*range(0, len(losses), 20), len(losses) - 1}):
        print("step %3d  squared error of the attention output %.3e" % (i, losses[i]))
    print("answers to one token of each request:", tuple(answer.shape))


if __name__ == "__main__":
    main()
