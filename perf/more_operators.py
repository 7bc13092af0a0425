"""Performance cases of the operators around a transformer block's projections: root-mean-square norm on the residual stream,
the gated feed-forward projections, linear layers trained from activations kept in 8 bits, and layers on 4-bit weights with a scale
per group.

A case is a dict of plain values.  `kind` names the operator:

  norm    `train` false: the stream's addition, the norm and its result in 8 bits; true: addition, norm and the gradients
  gated   `train` false: both projections, activation and product; true: that and the gradients, from what `keep` says was kept of the
          projections' results: values of the operator's type, or 8-bit blocks
  linear  a training step's part of a linear layer: its input is kept as 8-bit blocks, the gradients are made from these
  group   a layer on 4-bit weights in groups of 32 with a scale each

Blocks are 32 neighbouring elements of a row with one power of two as their scale, the least with which none is out of range.
Where `own` is false, run() computes the same in elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 32
E4M3_MAX = 448.0
E2M1_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # One new token of eight requests ahead of a quantized projection: the smallest call, latency.
        dict(name="norm_tokens", kind="norm", train=False, type="fp32", M=8, K=1280),
        # All pixels of the finest level at batch 8, in bf16, and codes for the quantized projection behind it: bytes.
        dict(name="norm_codes", kind="norm", train=False, type="bf16", M=32768, K=320),
        # A training step's norm of a wide stream, with the gradient of its weights over all rows.
        dict(name="norm_train", kind="norm", train=True, type="bf16", M=8192, K=5120),
        # A single token through a feed-forward block's projections: bound by the weights read.
        dict(name="gated_token", kind="gated", train=False, type="bf16", act="silu", keep="none", M=1, K=4096, N=10240),
        # The coarsest attention level at batch 8 in the type of the layers' results, exact GELU: ordinary.
        dict(name="gated_forward_fp32", kind="gated", train=False, type="fp32", act="gelu", keep="none", M=2048, K=1280, N=5120),
        # A training step of a wide block, what the backward pass needs kept in 8 bits: the largest piece of work.
        dict(name="gated_train", kind="gated", train=True, type="bf16", act="silu", keep="blocks", M=8192, K=1280, N=5120),
        # A short batch of odd length and odd widths, everything in fp32.
        dict(name="gated_train_odd_fp32", kind="gated", train=True, type="fp32", act="gelu", keep="type", M=999, K=333, N=1283),
        # A projection of the finest level at batch 8: many rows, few columns, the weights' gradient over a long axis.
        dict(name="linear_long", kind="linear", type="bf16", M=32768, K=320, N=960),
        # The output projection of a feed-forward block on a ragged batch.
        dict(name="linear_ragged", kind="linear", type="bf16", M=5003, K=5120, N=1280),
        # A new token on 4-bit weights: bound by the codes and scales read.
        dict(name="group_token", kind="group", type="bf16", M=1, K=5120, N=20480),
        # Sixteen requests' tokens with activations in fp32.
        dict(name="group_tokens_fp32", kind="group", type="fp32", M=16, K=5120, N=5120),
        # A prompt on the same kind of weights.
        dict(name="group_prompt", kind="group", type="bf16", M=2048, K=4096, N=4096),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _width(rng, lo, hi):
    """Network widths are multiples of 64 as a rule; some are odd."""
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.6 else n


def draw(rng):
    kind = rng.choice(["norm", "gated", "gated", "linear", "group", "group"])
    t = rng.choice(["bf16", "bf16", "fp32"])
    while True:
        if kind == "norm":
            c = dict(kind=kind, train=rng.random() < 0.5, type=t, M=_log(rng, 1, 65536), K=_width(rng, 32, 8192))
            if c["M"] * c["K"] <= 8192 * 5120:
                return c
        if kind == "gated":
            train = rng.random() < 0.6
            c = dict(kind=kind, train=train, type=t, act=rng.choice(["silu", "gelu"]), keep="none", M=_log(rng, 1, 16384), K=_width(rng, 32, 5120),
                     N=_width(rng, 32, 10240))
            if train:
                c["keep"] = rng.choice(["type", "blocks"]) if t == "bf16" else "type"
            if c["M"] * c["K"] * c["N"] <= 8192 * 1280 * 5120 and c["M"] * c["N"] <= 8192 * 5120:
                return c
        if kind == "linear":
            c = dict(kind=kind, type=t, M=_log(rng, 1, 32768), K=_width(rng, 32, 8192), N=_width(rng, 32, 8192))
            if c["M"] * c["K"] * c["N"] <= 8192 * 1280 * 5120 and c["M"] * (c["K"] + c["N"]) <= 8192 * 6400:
                return c
        if kind == "group":
            c = dict(kind=kind, type=t, M=rng.choice([_log(rng, 1, 16), _log(rng, 1, 2048)]), K=_width(rng, 32, 16384), N=_width(rng, 32, 20480))
            if c["N"] * c["K"] <= 5120 * 20480 and c["M"] * c["K"] * c["N"] <= 8192 * 1280 * 5120:
                return c


def _padded(n):
    return -(-n // BLOCK) * BLOCK


def work(c):
    s, M, K = 4 if c["type"] == "fp32" else 2, c["M"], c["K"]
    if c["kind"] == "norm":
        if c["train"]:                     # x, residual, and for the backward pass the stream and two gradients; the stream, y, a gradient
            return {"bytes": s * M * K * 8 + 8 * K + 8 * M, "flops": 14 * M * K}
        return {"bytes": s * M * K * 4 + M * K + 4 * K, "flops": 6 * M * K}
    N = c["N"]
    if c["kind"] == "gated":
        kept = {"none": 0, "type": s * 2 * N, "blocks": 2 * _padded(N) * 33 / 32}[c["keep"]]
        forward = s * (M * K + 2 * N * K + M * N) + M * kept
        if not c["train"]:
            return {"bytes": forward, "flops": 4 * M * N * K}
        return {"bytes": forward + M * kept + s * (M * N + 2 * M * K + 4 * N * K), "flops": 12 * M * N * K}
    if c["kind"] == "linear":
        blocks = M * _padded(K) * 33 / 32
        return {"bytes": s * (2 * M * K + M * N + 2 * N * K) + 2 * blocks + 4 * N, "flops": 4 * M * N * K}
    return {"bytes": s * M * (K + N) + N * _padded(K) * (1 / 2 + 1 / 32) + 4 * N, "flops": 2 * M * N * K}


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) + 1)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _activations(g, M, K):
    """Rows of different sizes, some channels larger than the others, as a network's hidden states are."""
    return _randn(g, M, K) * torch.exp(0.5 * _randn(g, M, 1)) * torch.exp(0.5 * _randn(g, K))


def _inputs(c, seed):
    g, t, M, K = _gen(seed), TYPES[c["type"]], c["M"], c["K"]
    if c["kind"] == "norm":
        s = {"x": _randn(g, M, K).to(t), "residual": _activations(g, M, K).to(t), "w": 1 + 0.2 * _randn(g, K)}
        if c["train"]:
            s["gy"], s["gs"] = _randn(g, M, K).to(t), _randn(g, M, K).to(t)
        else:
            # the static scale that calibration gave: values up to about four deviations are in range
            s["scale"] = torch.tensor([4.0 / E4M3_MAX], device=DEVICE)
        return s
    N = c["N"]
    if c["kind"] == "gated":
        s = {"x": _randn(g, M, K).to(t), "w": (_randn(g, 2 * N, K) * K ** -0.5).to(t), "bias": None}
        if c["type"] == "fp32":
            s["bias"] = 0.1 * _randn(g, 2 * N)
        if c["train"]:
            s["gh"] = _randn(g, M, N).to(t)
        return s
    if c["kind"] == "linear":
        return {"x": _activations(g, M, K).to(t), "w": (_randn(g, N, K) * K ** -0.5).to(t), "gy": _randn(g, M, N).to(t)}
    s = {"x": _randn(g, M, K).to(t), "bias": 0.1 * _randn(g, N)}
    s["codes"], s["scales"] = _pack4(_randn(g, N, K) * K ** -0.5 * torch.exp(0.3 * _randn(g, N, 1)))
    return s


def _pack4(w):
    """4-bit codes, the even element of a pair in the low half of a byte, and scales: done once, when the weights are loaded."""
    N, K = w.shape
    b = torch.nn.functional.pad(w, (0, _padded(K) - K)).view(N, -1, BLOCK)
    bits = b.abs().amax(2).view(torch.int32)
    e = (bits >> 23) - 2 + ((bits & 0x7fffff) > 0x400000).int()
    scales = torch.where(bits > 0, e.clamp(1, 254), 127)
    v = b * ((254 - scales) << 23).view(torch.float32)[:, :, None]
    # the upper of two neighbours from their middle on, from above it where the lower one is even
    middles = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEVICE)
    code = torch.bucketize(v.abs(), middles, right=False)
    tie = (v.abs()[..., None] == middles[1::2]).any(-1)
    code = (code + tie.long() + 8 * (v < 0).long()).to(torch.uint8).view(N, -1, 2)
    return (code[:, :, 0] | code[:, :, 1] << 4).contiguous(), scales.to(torch.uint8)


def prepare(c, seed):
    s = _inputs(c, seed)
    s["case"] = dict(c)
    if own:
        _results(c, s)
    return s


def _results(c, s):
    """Result buffers and workspaces, which a program keeps from step to step."""
    from paper_2408_06995_amd import binding as fpq

    def room(n):
        return torch.empty(max(int(n), 256), dtype=torch.uint8, device=DEVICE)

    def like(k):
        return torch.empty_like(s[k])

    M, K, N, t = c["M"], c["K"], c.get("N"), fpq.FPQ_TYPE_FP32 if c["type"] == "fp32" else fpq.FPQ_TYPE_BF16
    if c["kind"] == "norm":
        s["sum"], s["y"] = like("x"), like("x")
        if c["train"]:
            s["rstd"], s["gx"], s["gw"] = torch.empty(M, device=DEVICE), like("x"), like("w")
            s["ws"] = room(fpq.fpq_rms_norm_backward_workspace_size(M, K))
        else:
            s["yq"] = torch.empty(M, fpq.fpq_padded_channels(K), dtype=torch.uint8, device=DEVICE)
    elif c["kind"] == "gated":
        s["h"], s["pre"], s["pre_scales"] = torch.empty(M, N, dtype=TYPES[c["type"]], device=DEVICE), None, None
        if c["keep"] == "type":
            s["pre"] = torch.empty(M, 2 * N, dtype=TYPES[c["type"]], device=DEVICE)
        elif c["keep"] == "blocks":
            n = M * 2 * _padded(N)
            s["pre"], s["pre_scales"] = room(n)[:n].view(M, -1), room(n // BLOCK)[:n // BLOCK].view(M, -1)
        s["ws"] = room(fpq.fpq_gated_workspace_size(M, N, K, t))
        if c["train"]:
            s["gx"], s["gw"] = like("x"), like("w")
            s["gb"] = like("bias") if s["bias"] is not None else None
            s["ws_backward"] = room(fpq.fpq_gated_backward_workspace_size(M, N, K, t))
    elif c["kind"] == "linear":
        s["xq"], s["xq_scales"] = room(M * _padded(K))[:M * _padded(K)].view(M, -1), room(M * _padded(K) // BLOCK)[:M * _padded(K) // BLOCK].view(M, -1)
        s["gx"], s["gw"], s["gb"] = like("x"), like("w"), torch.empty(N, device=DEVICE)
        s["ws"] = room(fpq.fpq_linear_backward_workspace_size(M, N, K, t))
    else:
        s["y"] = torch.empty(M, N, dtype=TYPES[c["type"]], device=DEVICE)
        s["ws"] = room(fpq.fpq_block_linear_workspace_size(M, N, K, t))


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"norm": _own_norm, "gated": _own_gated, "linear": _own_linear, "group": _own_group}[kind](s)
    return {"norm": _plain_norm, "gated": _plain_gated, "linear": _plain_linear, "group": _plain_group}[kind](s)


def _own_norm(s):
    from paper_2408_06995_amd import binding as fpq
    if not s["case"]["train"]:
        fpq.fpq_rms_norm(s["x"], s["residual"], s["w"], EPS, s["sum"], s["y"], None, s["yq"], (4, 3, 7, E4M3_MAX), 0.0, s["scale"])
        return {"sum": s["sum"], "y": s["y"], "yq": s["yq"][:, :s["case"]["K"]].view(torch.float8_e4m3fn)}
    fpq.fpq_rms_norm(s["x"], s["residual"], s["w"], EPS, s["sum"], s["y"], s["rstd"])
    fpq.fpq_rms_norm_backward(s["sum"], s["w"], s["rstd"], s["gy"], s["gs"], s["gx"], s["gw"], s["ws"])
    return {"sum": s["sum"], "y": s["y"], "gx": s["gx"], "gw": s["gw"]}


def _plain_norm(s):
    t = TYPES[s["case"]["type"]]
    total = (s["x"].float() + s["residual"].float()).to(t)
    r = total.float()                                                 # the norm is of the stream as it is kept
    rstd = 1 / torch.sqrt((r * r).mean(1, keepdim=True) + EPS)
    y = r * rstd * s["w"]
    if not s["case"]["train"]:
        q = (y * (1 / s["scale"])).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        return {"sum": total, "y": y.to(t), "yq": q}
    gy = s["gy"].float()
    g = gy * s["w"]
    gx = rstd * (g - r * (rstd * rstd * (g * r).mean(1, keepdim=True))) + s["gs"].float()
    return {"sum": total, "y": y.to(t), "gx": gx.to(t), "gw": (gy * r * rstd).sum(0)}


def _own_gated(s):
    from paper_2408_06995_amd import binding as fpq
    c = s["case"]
    act = fpq.FPQ_GATE_SILU if c["act"] == "silu" else fpq.FPQ_GATE_GELU
    fpq.fpq_gated(s["x"], s["w"], s["bias"], act, s["h"], s["pre"], s["pre_scales"], s["ws"])
    if not c["train"]:
        return {"h": s["h"]}
    fpq.fpq_gated_backward(s["x"], None, s["w"], s["pre"], s["pre_scales"], act, s["gh"], s["gx"], s["gw"], s["gb"], s["ws_backward"])
    out = {"h": s["h"], "gx": s["gx"], "gw": s["gw"]}
    if c["keep"] == "blocks":
        out["pre"] = s["pre"].view(torch.float8_e4m3fn)
    if s["gb"] is not None:
        out["gb"] = s["gb"]
    return out


def _gate(g, act):
    """The activation and its derivative."""
    if act == "silu":
        z = 1 / (1 + torch.exp(-g))
        return g * z, z * (1 + g * (1 - z))
    z = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
    return g * z, z + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5


def _blocks8(x):
    """E4M3 codes [M, padded columns] and scales of rows, and the values that they stand for."""
    M, K = x.shape
    b = torch.nn.functional.pad(x, (0, _padded(K) - K)).view(M, -1, BLOCK)
    bits = b.abs().amax(2).view(torch.int32)
    e = (bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000).int()
    scales = torch.where(bits > 0, e.clamp(1, 254), 127)
    codes = (b * ((254 - scales) << 23).view(torch.float32)[:, :, None]).to(torch.float8_e4m3fn)
    values = codes.float() * (scales << 23).view(torch.float32)[:, :, None]
    return codes.view(M, -1), scales.to(torch.uint8), values.view(M, -1)[:, :K]


def _plain_gated(s):
    c = s["case"]
    t, N = TYPES[c["type"]], c["N"]
    x, w = s["x"].float(), s["w"].float()
    pre = torch.matmul(x, w.t())
    if s["bias"] is not None:
        pre = pre + s["bias"]
    a, g = pre[:, :N], pre[:, N:]
    out = {"h": (a * _gate(g, c["act"])[0]).to(t)}
    if not c["train"]:
        return out
    if c["keep"] == "blocks":
        (qa, _, a), (qg, _, g) = _blocks8(a), _blocks8(g)
        out["pre"] = torch.cat([qa.view(torch.uint8), qg.view(torch.uint8)], 1).view(torch.float8_e4m3fn)
    else:
        a, g = a.to(t).float(), g.to(t).float()
    gh = s["gh"].float()
    f, df = _gate(g, c["act"])
    d = torch.cat([gh * f, gh * a * df], 1)
    out["gx"], out["gw"] = torch.matmul(d, w).to(t), torch.matmul(d.t(), x).to(t)
    if s["bias"] is not None:
        out["gb"] = d.sum(0)
    return out


def _own_linear(s):
    from paper_2408_06995_amd import binding as fpq
    fpq.fpq_block_quantize(s["x"], (4, 3, 7, E4M3_MAX), None, s["xq"], s["xq_scales"])
    fpq.fpq_linear_backward(s["xq"], s["xq_scales"], s["w"], s["gy"], s["gx"], s["gw"], s["gb"], s["ws"])
    return {"xq": s["xq"].view(torch.float8_e4m3fn), "xq_scales": s["xq_scales"], "gx": s["gx"], "gw": s["gw"], "gb": s["gb"]}


def _plain_linear(s):
    t = TYPES[s["case"]["type"]]
    codes, scales, x = _blocks8(s["x"].float())
    gy = s["gy"].float()
    return {"xq": codes, "xq_scales": scales, "gx": torch.matmul(gy, s["w"].float()).to(t), "gw": torch.matmul(gy.t(), x).to(t), "gb": gy.sum(0)}


def _own_group(s):
    from paper_2408_06995_amd import binding as fpq
    fpq.fpq_block_linear(s["x"], s["codes"], s["scales"], s["bias"], s["y"], s["ws"])
    return {"y": s["y"]}


def _plain_group(s):
    c = s["case"]
    values = torch.tensor(E2M1_VALUES + [-v for v in E2M1_VALUES], device=DEVICE)
    code = torch.stack([s["codes"] & 15, s["codes"] >> 4], 2).int()
    scale = (s["scales"].int() << 23).view(torch.float32)
    w = (values[code].view(c["N"], -1, BLOCK) * scale[:, :, None]).view(c["N"], -1)[:, :c["K"]]
    return {"y": (torch.matmul(s["x"].float(), w.t()) + s["bias"]).to(TYPES[c["type"]])}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(c, seed):
    return {"norm": _exact_norm, "gated": _exact_gated, "linear": _exact_linear, "group": _exact_group}[c["kind"]](c, seed)


def _exact_norm(c, seed):
    """The codes are choices between neighbours, which have no value of their own in 64 bits."""
    s = _inputs(c, seed)
    total = s["x"].double() + s["residual"].double()
    r, w = total.to(TYPES[c["type"]]).double(), s["w"].double()
    norm = r / torch.sqrt(torch.sum(r ** 2, 1, keepdim=True) / c["K"] + EPS)
    if not c["train"]:
        return {"sum": total, "y": norm * w, "yq": None}
    rms = torch.sqrt(torch.sum(r ** 2, 1, keepdim=True) / c["K"] + EPS)
    gn = s["gy"].double() * w
    gr = (gn - norm * torch.sum(gn * norm, 1, keepdim=True) / c["K"]) / rms
    return {"sum": total, "y": norm * w, "gx": gr + s["gs"].double(), "gw": torch.sum(s["gy"].double() * norm, 0)}


def _pow2(e):
    return (e.long() + 1023 << 52).view(torch.float64)


def _e4m3_blocks(x):
    """(codes' values, exponents, values) of the nearest E4M3 numbers in units of each block's scale."""
    M, K = x.shape
    b = torch.zeros(M, _padded(K), dtype=torch.float64, device=DEVICE)
    b[:, :K] = x
    b = b.view(M, -1, BLOCK)
    m, e = torch.frexp(b.abs().amax(2))                              # the largest is m 2^e, 0.5 <= m < 1
    e = torch.where(m == 0, 0, torch.where(m <= 0.875, e - 9, e - 8)).clamp(-126)
    v = b * _pow2(-e[:, :, None])
    step = _pow2(torch.frexp(v)[1].clamp(-5) - 4)
    v = torch.round(v / step) * step
    return v.view(M, -1), e, (v * _pow2(e[:, :, None])).view(M, -1)[:, :K]


def _exact_gated(c, seed):
    """What the forward pass keeps is part of the definition: rounded to its type, or the blocks' values.  The codes themselves are
    choices between neighbours."""
    s = _inputs(c, seed)
    x, w = s["x"].double(), s["w"].double()
    pre = x @ w.T
    if s["bias"] is not None:
        pre += s["bias"].double()

    def gate(g):
        if c["act"] == "silu":
            p = torch.special.expit(g)
            return g * p, p + g * p * (1 - p)
        p = torch.special.ndtr(g)
        return g * p, p + g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)

    a, g = torch.split(pre, c["N"], dim=1)
    out = {"h": a * gate(g)[0]}
    if not c["train"]:
        return out
    if c["keep"] == "blocks":
        out["pre"] = None
        a, g = _e4m3_blocks(a)[2], _e4m3_blocks(g)[2]
    else:
        a, g = (v.to(TYPES[c["type"]]).double() if c["type"] == "bf16" else v for v in (a, g))
    gh = s["gh"].double()
    value, slope = gate(g)
    da, dg = gh * value, gh * a * slope
    out["gx"] = da @ w[:c["N"]] + dg @ w[c["N"]:]
    out["gw"] = torch.cat([da.T @ x, dg.T @ x])
    if s["bias"] is not None:
        out["gb"] = torch.cat([torch.sum(da, 0), torch.sum(dg, 0)])
    return out


def _exact_linear(c, seed):
    s = _inputs(c, seed)
    gy = s["gy"].double()
    codes, _, x = _e4m3_blocks(s["x"].double())
    return {"xq": codes, "xq_scales": None, "gx": gy @ s["w"].double(), "gw": gy.T @ x, "gb": torch.sum(gy, 0)}


def _exact_group(c, seed):
    s = _inputs(c, seed)
    low, high = s["codes"] % 16, s["codes"] // 16
    code = torch.stack((low, high), 2).view(c["N"], -1).long()
    exponent, mantissa = code // 2 % 4, code % 2
    w = torch.where(exponent == 0, 0.5 * mantissa.double(), (1 + 0.5 * mantissa.double()) * _pow2(exponent - 1))
    w = torch.where(code >= 8, -w, w) * torch.repeat_interleave(_pow2(s["scales"].long() - 127), BLOCK, dim=1)
    return {"y": s["x"].double() @ w[:, :c["K"]].T + s["bias"].double()}
