"""Performance cases of the operators for adapting a quantized U-Net: attention and its gradient, low-rank adapters of many
requests beside a shared projection and their gradients, AdamW over many tensors.

A case is a dict of plain values.  `kind` names the operator:

  attention  `train` false: the forward pass; true: forward and backward, as a training step makes them
  adapter    `train` false: y += adapters(x) for the rows of many requests; true: that and the gradients
  adamw      one optimizer step over all tensors of a set

Where `own` is false, run() computes the same in elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 256                   # elements of a tensor that share the scales of their 8-bit states
E4M3_MAX = 448.0
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # One new token per sample over caches of different lengths, four query heads on each key head: serving, bound by
        # the keys and values read.
        dict(name="token_long_cache", kind="attention", train=False, type="bf16", B=16, Hq=32, Hkv=8, D=128, Lq=1, Lk=4096, causal=True, ragged=True),
        # The self-attention of the coarsest level of a U-Net at batch 1: the smallest call, latency.
        dict(name="middle_64", kind="attention", train=False, type="fp32", B=1, Hq=8, Hkv=8, D=160, Lq=64, Lk=64, causal=False, ragged=False),
        # Cross-attention of the finest level at batch 8: every pixel over 77 text tokens, of which a sample uses some.
        dict(name="context_77", kind="attention", train=False, type="fp32", B=8, Hq=8, Hkv=8, D=40, Lq=4096, Lk=77, causal=False, ragged=True),
        # Self-attention of the finest level at batch 4, a training step in bf16: the largest piece of work.
        dict(name="train_4096", kind="attention", train=True, type="bf16", B=4, Hq=8, Hkv=8, D=40, Lq=4096, Lk=4096, causal=False, ragged=False),
        # Self-attention of the second level at batch 2, a training step in the type of the layers' results.
        dict(name="train_1024_fp32", kind="attention", train=True, type="fp32", B=2, Hq=8, Hkv=8, D=80, Lq=1024, Lk=1024, causal=False, ragged=False),
        # A text model's causal layer with shared key heads and samples of different odd lengths, a training step.
        dict(name="train_causal_shared", kind="attention", train=True, type="bf16", B=4, Hq=16, Hkv=4, D=128, Lq=1999, Lk=1999, causal=True, ragged=True),
        # Time-embedding projections of 64 requests, one row and one adapter each: latency.
        dict(name="adapter_rows", kind="adapter", train=False, x="fp32", w="bf16", K=1280, N=1280, R=16, adapters=64, requests=64, rows=64),
        # An attention output projection of the finest level, eight images in five styles: ordinary serving.
        dict(name="adapter_images", kind="adapter", train=False, x="fp32", w="bf16", K=320, N=320, R=16, adapters=5, requests=8, rows=32768),
        # The query / key / value projection of the finest level at batch 4, two adapters in training.
        dict(name="adapter_train_qkv", kind="adapter", train=True, x="fp32", w="fp32", K=320, N=960, R=16, adapters=2, requests=4, rows=16384),
        # A wide projection, a higher rank, requests of odd lengths that share nine adapters, all in bf16.
        dict(name="adapter_train_ragged", kind="adapter", train=True, x="bf16", w="bf16", K=1280, N=5120, R=64, adapters=9, requests=37, rows=5003),
        # The adapters of a U-Net's attention projections (16 blocks, eight projections each): many small tensors, with the
        # copies in bf16 that the layers read.
        dict(name="adamw_adapters", kind="adamw", tensors=256, largest=1280 * 16, state=32, param="fp32", grad="fp32", copy=True),
        # Rounding parameters of whole layers, as many as weights: 8-bit states.
        dict(name="adamw_rounding_8bit", kind="adamw", tensors=40, largest=1280 * 5120, state=8, param="fp32", grad="fp32", copy=False),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "attention", "adapter", "adapter", "adapter", "adamw"])
    if kind == "attention":
        while True:
            Hkv = rng.choice([1, 2, 4, 8])
            c = dict(kind=kind, train=rng.random() < 0.5, type=rng.choice(["fp32", "bf16"]), B=_log(rng, 1, 16), Hkv=Hkv,
                     Hq=Hkv * rng.choice([1, 1, 1, 2, 4]), D=rng.choice([40, 64, 80, 96, 128, 160, rng.randint(8, 160)]), causal=rng.random() < 0.4,
                     ragged=rng.random() < 0.4)
            c["Lq"] = _log(rng, 1, 4096)
            c["Lk"] = rng.choice([c["Lq"], _log(rng, 1, 4096)])
            if c["B"] * c["Hq"] * c["Lq"] * c["Lk"] * c["D"] <= 32 * 4096 * 4096 * 40:
                return c
    if kind == "adapter":
        while True:
            x = rng.choice(["fp32", "fp32", "bf16"])
            c = dict(kind=kind, train=rng.random() < 0.5, x=x, w=rng.choice(["fp32", "bf16"]) if x == "fp32" else "bf16", K=_log(rng, 64, 5120),
                     N=_log(rng, 64, 5120), R=rng.choice([4, 8, 16, 32, 64, rng.randint(1, 128)]), adapters=_log(rng, 1, 32), requests=_log(rng, 1, 128))
            if rng.random() < 0.6:                       # network widths are multiples of 64 as a rule
                c["K"], c["N"] = c["K"] // 64 * 64, c["N"] // 64 * 64
            c["rows"] = max(c["requests"], _log(rng, 1, 32768))
            if c["rows"] * (c["K"] + c["N"]) <= 32768 * 1280 and c["rows"] * c["adapters"] * c["R"] * (c["K"] + c["N"]) <= 1 << 38:
                return c
    while True:
        c = dict(kind=kind, tensors=_log(rng, 1, 400), largest=_log(rng, 64, 1280 * 5120), state=rng.choice([32, 8]), param=rng.choice(["fp32", "fp32", "bf16"]),
                 grad=rng.choice(["fp32", "fp32", "bf16"]), copy=False)
        c["copy"] = c["param"] == "fp32" and rng.random() < 0.5
        if sum(_sizes(c)) <= 80 << 20:
            return c


# ------------------------------------------------------------------------------------------------ what a case holds

def _lens(c):
    """Keys of each sample: half to all of the buffer, and none in the last of four or more samples (a request without text)."""
    if not c["ragged"]:
        return [c["Lk"]] * c["B"]
    n = [max(1, c["Lk"] - (b * 37 % 16) * c["Lk"] // 32) for b in range(c["B"])]
    if c["B"] >= 4:
        n[-1] = 0
    return n


def _visible(c, n):
    """Pairs of a query and a key of one head of a sample of n keys; under `causal` the last query sees all keys."""
    if not c["causal"]:
        return c["Lq"] * n
    return sum(max(0, min(n, i + n - c["Lq"] + 1)) for i in range(c["Lq"]))


def _sizes(c):
    """Elements of each tensor: the largest, and others down to a hundredth of it, odd ones among them."""
    return [max(1, int(c["largest"] * 0.01 ** ((i * 7 % c["tensors"]) / c["tensors"]))) for i in range(c["tensors"])]


def _starts(c):
    """First row of each request, and the end: near-equal lengths, of which every other lends its neighbour a third."""
    n, q = c["requests"], c["rows"] // c["requests"]
    at = [r * c["rows"] // n for r in range(n + 1)]
    return [v + (q // 3 if r % 2 and r < n else 0) for r, v in enumerate(at)]


def _adapter_of(c):
    """The adapter of each request; the last of eight or more requests has none."""
    of = [(r * 5 + 1) % c["adapters"] for r in range(c["requests"])]
    if c["requests"] >= 8:
        of[-1] = -1
    return of


def work(c):
    if c["kind"] == "attention":
        size = 4 if c["type"] == "fp32" else 2
        lens = _lens(c)
        q, kv = c["B"] * c["Lq"] * c["Hq"] * c["D"], 2 * sum(lens) * c["Hkv"] * c["D"]
        pairs = c["Hq"] * sum(_visible(c, n) for n in lens)
        if not c["train"]:
            return {"bytes": size * (2 * q + kv) + 4 * c["B"] * c["Hq"] * c["Lq"], "flops": 4 * pairs * c["D"]}
        kv_all = 2 * c["B"] * c["Lk"] * c["Hkv"] * c["D"]
        return {"bytes": size * (4 * q + kv + kv_all) + 4 * c["B"] * c["Hq"] * c["Lq"], "flops": 14 * pairs * c["D"]}
    if c["kind"] == "adapter":
        xs, ws = (4 if c[t] == "fp32" else 2 for t in ("x", "w"))
        used = len({a for a in _adapter_of(c) if a >= 0})
        M, K, N, R = c["rows"], c["K"], c["N"], c["R"]
        forward = xs * M * (K + 2 * N) + ws * used * R * (K + N) + 4 * M * R
        if not c["train"]:
            return {"bytes": forward, "flops": 2 * M * R * (K + N)}
        return {"bytes": forward + xs * M * (N + 2 * K) + 4 * c["adapters"] * R * (K + N), "flops": 6 * M * R * (K + N)}
    n = sum(_sizes(c))
    each = 2 * (4 if c["param"] == "fp32" else 2) + (4 if c["grad"] == "fp32" else 2) + (2 if c["copy"] else 0)
    each += 16 if c["state"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * each, "flops": 14 * n}


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) + 1)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _attention_inputs(c, seed):
    g, t = _gen(seed), TYPES[c["type"]]
    s = {"scale": c["D"] ** -0.5, "lens": _ints(_lens(c)) if c["ragged"] else None}
    if c["Lq"] == c["Lk"]:
        # self-attention: queries, keys and values are columns of one projection's result
        qkv = (_randn(g, c["B"], c["Lq"], c["Hq"] + 2 * c["Hkv"], c["D"])).to(t)
        s["q"], s["k"], s["v"] = qkv.split([c["Hq"], c["Hkv"], c["Hkv"]], dim=2)
    else:
        s["q"] = _randn(g, c["B"], c["Lq"], c["Hq"], c["D"]).to(t)
        s["k"], s["v"] = (_randn(g, c["B"], c["Lk"], c["Hkv"], c["D"]).to(t) for _ in range(2))
    s["go"] = _randn(g, c["B"], c["Lq"], c["Hq"], c["D"]).to(t) if c["train"] else None
    return s


def _adapter_inputs(c, seed):
    g, tx, tw = _gen(seed), TYPES[c["x"]], TYPES[c["w"]]
    M, K, N, R, n = (c[v] for v in ("rows", "K", "N", "R", "adapters"))
    # y0, gx0: what the shared projection gives, forward and backward
    s = {"x": _randn(g, M, K).to(tx), "y0": _randn(g, M, N).to(tx), "a": (_randn(g, n, R, K) * K ** -0.5).to(tw), "b": (_randn(g, n, N, R) * 0.1).to(tw),
         "scaling": torch.rand(n, generator=g, device=DEVICE) + 0.5, "row_start": _ints(_starts(c)), "adapter": _ints(_adapter_of(c))}
    if c["train"]:
        s["gy"], s["gx0"] = _randn(g, M, N).to(tx), _randn(g, M, K).to(tx)
    return s


def _adamw_inputs(c, seed):
    """All tensors of a kind in one buffer, each from a multiple of a block on: (first, elements) of each in "at"."""
    g = _gen(seed)
    at, n = [], 0
    for size in _sizes(c):
        at.append((n, size))
        n += -(-size // BLOCK) * BLOCK
    inside = torch.zeros(n, dtype=torch.bool, device=DEVICE)
    first, size = (torch.tensor(v, device=DEVICE) for v in zip(*at))
    owner = torch.repeat_interleave(torch.arange(len(at), device=DEVICE), -(-size // BLOCK) * BLOCK, output_size=n)
    inside = torch.arange(n, device=DEVICE) - first[owner] < size[owner]
    spread = torch.exp2(_randn(g, n // BLOCK, 1)).expand(-1, BLOCK).reshape(-1) * 1e-3      # layers' gradients differ in size
    m = _randn(g, n) * spread * inside
    v = (_randn(g, n) * spread).square() * 0.5 * inside + m * m
    s = {"at": at, "param": (_randn(g, n) * 0.05 * inside).to(TYPES[c["param"]]), "grad": (_randn(g, n) * 2 * spread * inside).to(TYPES[c["grad"]]), "step": 10}
    if c["state"] == 32:
        s["m"], s["v"] = m, v
    else:
        for k, x in (("m", m), ("v", v.sqrt())):
            top = x.abs().view(-1, BLOCK).amax(1)
            s[k + "_scale"] = torch.where(top > 0, top / E4M3_MAX, torch.ones_like(top))
            s[k] = (x.view(-1, BLOCK) / s[k + "_scale"][:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(-1)
    s["copy"] = s["param"].to(torch.bfloat16) if c["copy"] else None
    return s


def prepare(c, seed):
    s = {"attention": _attention_inputs, "adapter": _adapter_inputs, "adamw": _adamw_inputs}[c["kind"]](c, seed)
    s["case"] = dict(c)
    if own:
        _results(c, s)
    return s


def _results(c, s):
    """Result buffers, workspaces and the optimizer's plan, which a program keeps from step to step."""
    from paper_2408_06995_amd import binding as fpq

    def room(n):
        return torch.empty(max(int(n), 256), dtype=torch.uint8, device=DEVICE)

    if c["kind"] == "attention":
        sizes = (c["B"], c["Hq"], c["Hkv"], c["Lq"], c["Lk"], c["D"], fpq.FPQ_TYPE_FP32 if c["type"] == "fp32" else fpq.FPQ_TYPE_BF16)
        s["o"] = torch.empty_like(s["q"], memory_format=torch.contiguous_format)
        s["lse"] = torch.empty(c["B"], c["Hq"], c["Lq"], device=DEVICE)
        s["ws"] = room(fpq.fpq_attention_workspace_size(*sizes))
        if c["train"]:
            s["grads"] = [torch.empty_like(s[k], memory_format=torch.contiguous_format) for k in "qkv"]
            s["ws_backward"] = room(fpq.fpq_attention_backward_workspace_size(*sizes))
    elif c["kind"] == "adapter":
        sizes = (c["rows"], c["N"], c["K"], c["R"], c["requests"], c["adapters"])
        s["y"], s["t"] = torch.empty_like(s["y0"]), torch.empty(c["rows"], c["R"], device=DEVICE)
        s["ws"] = room(fpq.fpq_adapter_workspace_size(*sizes))
        if c["train"]:
            s["gx"] = torch.empty_like(s["gx0"])
            s["ga"], s["gb"] = (torch.empty(s[k].shape, device=DEVICE) for k in "ab")
            s["ws_backward"] = room(fpq.fpq_adapter_backward_workspace_size(*sizes))
    else:
        items = []
        for first, size in s["at"]:
            part = [s[k][first:first + size] for k in ("param", "grad", "m", "v")]
            scales = [s[k][first // BLOCK:-(-(first + size) // BLOCK)] if c["state"] == 8 else None for k in ("m_scale", "v_scale")]
            items.append((*part, *scales, s["copy"][first:first + size] if c["copy"] else None))
        s["tensors"] = fpq.adamw_tensors(items)
        s["plan"] = room(fpq.fpq_adamw_plan_size(s["tensors"]))
        s["info"] = fpq.fpq_adamw_plan(s["tensors"], s["plan"])


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"attention": _own_attention, "adapter": _own_adapter, "adamw": _own_adamw}[kind](s)
    return {"attention": _plain_attention, "adapter": _plain_adapter, "adamw": _plain_adamw}[kind](s)


def _own_attention(s):
    from paper_2408_06995_amd import binding as fpq
    causal = int(s["case"]["causal"])
    fpq.fpq_attention(s["q"], s["k"], s["v"], s["o"], s["lse"], s["scale"], causal, s["lens"], s["ws"])
    if s["go"] is None:
        return {"o": s["o"], "lse": s["lse"]}
    fpq.fpq_attention_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["go"], *s["grads"], s["scale"], causal, s["lens"], s["ws_backward"])
    return {"o": s["o"], "lse": s["lse"], "gq": s["grads"][0], "gk": s["grads"][1], "gv": s["grads"][2]}


def _plain_attention(s):
    c = s["case"]
    t, B, Hkv, G, Lq, Lk, D = TYPES[c["type"]], c["B"], c["Hkv"], c["Hq"] // c["Hkv"], c["Lq"], c["Lk"], c["D"]

    def heads(x, n):                                                  # [B, L, Hkv * n, D] -> [B, Hkv, n, L, D]
        return x.float().view(B, -1, Hkv, n, D).permute(0, 2, 3, 1, 4).contiguous()

    def tokens(x):                                                    # and back
        return x.permute(0, 3, 1, 2, 4).reshape(B, x.shape[3], -1, D).to(t)

    q, k, v = heads(s["q"], G), heads(s["k"], 1), heads(s["v"], 1)
    lens = s["lens"] if s["lens"] is not None else torch.full((B,), Lk, device=DEVICE)
    i, j = torch.arange(Lq, device=DEVICE)[:, None], torch.arange(Lk, device=DEVICE)
    seen = j < lens[:, None, None]
    if c["causal"]:
        seen = seen & (j <= i + lens[:, None, None] - Lq)
    seen = seen[:, None, None]
    x = torch.matmul(q, k.transpose(-1, -2)) * s["scale"]
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    some = top > -math.inf
    p = torch.exp(x - torch.where(some, top, 0.0))
    total = p.sum(-1, keepdim=True)
    p = torch.where(some, p / total, 0.0)
    o = torch.matmul(p, v)
    lse = (top + torch.log(total)).view(B, Hkv * G, Lq)
    if s["go"] is None:
        return {"o": tokens(o), "lse": lse}
    go = heads(s["go"], G)
    gv = torch.matmul(p.transpose(-1, -2), go).sum(2, keepdim=True)
    ds = p * (torch.matmul(go, v.transpose(-1, -2)) - (go * o).sum(-1, keepdim=True)) * s["scale"]
    gq = torch.matmul(ds, k)
    gk = torch.matmul(ds.transpose(-1, -2), q).sum(2, keepdim=True)
    return {"o": tokens(o), "lse": lse, "gq": tokens(gq), "gk": tokens(gk), "gv": tokens(gv)}


def _own_adapter(s):
    from paper_2408_06995_amd import binding as fpq
    common = (s["x"], s["a"], s["b"], s["scaling"], s["row_start"], s["adapter"])
    fpq.fpq_adapter_apply(*common, s["y0"], s["y"], s["t"], s["ws"])
    if not s["case"]["train"]:
        return {"y": s["y"]}
    fpq.fpq_adapter_backward(*common, s["t"], s["gy"], s["gx0"], s["gx"], s["ga"], s["gb"], s["ws_backward"])
    return {"y": s["y"], "gx": s["gx"], "ga": s["ga"], "gb": s["gb"]}


def _plain_adapter(s):
    c = s["case"]
    M, K, N, R, n, t = c["rows"], c["K"], c["N"], c["R"], c["adapters"], TYPES[c["x"]]
    x, a, b = s["x"].float(), s["a"].float().view(n * R, K), s["b"].float().permute(1, 0, 2).reshape(N, n * R)
    request = torch.searchsorted(s["row_start"], torch.arange(M, device=DEVICE, dtype=torch.int32), right=True) - 1
    of = s["adapter"][request]
    # every row through every adapter, and zero for all but the row's own
    mine = (of[:, None] == torch.arange(n, device=DEVICE)).float() * s["scaling"]
    mine = mine[:, :, None].expand(-1, -1, R).reshape(M, n * R)
    h = torch.matmul(x, a.t()) * mine
    y = (s["y0"].float() + torch.matmul(h, b.t())).to(t)
    if not c["train"]:
        return {"y": y}
    gy = s["gy"].float()
    gh = torch.matmul(gy, b) * mine
    gx = (s["gx0"].float() + torch.matmul(gh, a)).to(t)
    ga = torch.matmul(gh.t(), x).view(n, R, K)
    gb = torch.matmul(gy.t(), h).view(N, n, R).permute(1, 0, 2).contiguous()
    return {"y": y, "gx": gx, "ga": ga, "gb": gb}


def _state(s):
    return {k: s[k] for k in ("param", "m", "v", "m_scale", "v_scale", "copy") if s.get(k) is not None}


def _own_adamw(s):
    from paper_2408_06995_amd import binding as fpq
    s["step"] += 1
    fpq.fpq_adamw_step(s["plan"], s["info"], HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], HYPER["weight_decay"], s["step"])
    return _state(s)


def _plain_adamw(s):
    c, h = s["case"], HYPER
    s["step"] += 1
    g, p = s["grad"].float(), s["param"].float()
    m, root = s["m"].float(), s["v"].float()
    if c["state"] == 8:
        m = (m.view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        root = (root.view(-1, BLOCK) * s["v_scale"][:, None]).view(-1)
        root = root * root
    m = m * h["beta1"] + g * (1 - h["beta1"])
    v = root * h["beta2"] + g * (1 - h["beta2"]) * g
    root = torch.sqrt(v)
    update = m / (root * (1 - h["beta2"] ** s["step"]) ** -0.5 + h["eps"])
    p = p * (1 - h["lr"] * h["weight_decay"]) - update * (h["lr"] / (1 - h["beta1"] ** s["step"]))
    s["param"].copy_(p)
    if c["copy"]:
        s["copy"].copy_(p)
    if c["state"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return _state(s)
    m, root = m.view(-1, BLOCK), root.view(-1, BLOCK)
    for k, x in (("m", m), ("v", root)):
        top = x.abs().amax(1)
        scale = torch.where(top > 0, top / E4M3_MAX, 1.0)
        code = (x * (1 / scale)[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
        if k == "v":                                                  # a positive root stays one
            code = torch.where(x > 0, code.clamp(min=2.0 ** -9), code)
        s[k].copy_(code.to(torch.float8_e4m3fn).view(-1))
        s[k + "_scale"].copy_(scale)
    return _state(s)


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(c, seed):
    return {"attention": _exact_attention, "adapter": _exact_adapter, "adamw": _exact_adamw}[c["kind"]](c, seed)


def _exact_attention(c, seed):
    s = _attention_inputs(c, seed)
    q, k, v = (s[n].double() for n in "qkv")
    go = s["go"].double() if c["train"] else None
    o, gq, gk, gv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    lse = torch.full((c["B"], c["Hq"], c["Lq"]), -math.inf, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(_lens(c)):
        first = max(0, c["Lq"] - n) if c["causal"] else 0             # queries before it see no key
        if n == 0:
            continue
        for h in range(c["Hq"]):
            hk = h * c["Hkv"] // c["Hq"]
            Q, K, V = q[b, first:, h], k[b, :n, hk], v[b, :n, hk]
            S = (Q @ K.T) * s["scale"]
            if c["causal"]:
                S += torch.full_like(S, -math.inf).triu(n - c["Lq"] + first + 1)
            lse[b, h, first:] = torch.logsumexp(S, 1)
            P = torch.softmax(S, 1)
            o[b, first:, h] = P @ V
            if c["train"]:
                G = go[b, first:, h]
                dP = G @ V.T
                dS = P * (dP - (dP * P).sum(1, keepdim=True)) * s["scale"]
                gq[b, first:, h] = dS @ K
                gk[b, :n, hk] += dS.T @ Q
                gv[b, :n, hk] += P.T @ G
    return {"o": o, "lse": lse, "gq": gq, "gk": gk, "gv": gv} if c["train"] else {"o": o, "lse": lse}


def _exact_adapter(c, seed):
    s = _adapter_inputs(c, seed)
    x, y, a, b = (s[k].double() for k in ("x", "y0", "a", "b"))
    ga, gb = torch.zeros_like(a), torch.zeros_like(b)
    gy, gx = (s["gy"].double(), s["gx0"].double()) if c["train"] else (None, None)
    starts = _starts(c)
    for r, i in enumerate(_adapter_of(c)):
        if i < 0:
            continue
        rows, scale = slice(starts[r], starts[r + 1]), float(s["scaling"][i])
        t = x[rows] @ a[i].T
        y[rows] += scale * (t @ b[i].T)
        if c["train"]:
            gt = scale * (gy[rows] @ b[i])
            gx[rows] += gt @ a[i]
            ga[i] += gt.T @ x[rows]
            gb[i] += scale * (gy[rows].T @ t)
    return {"y": y, "gx": gx, "ga": ga, "gb": gb} if c["train"] else {"y": y}


def _exact_adamw(c, seed):
    """The codes of 8-bit states are choices between neighbours, which have no value of their own in 64 bits; their scales have."""
    s, h = _adamw_inputs(c, seed), HYPER
    t = s["step"] + 1
    g, p, m, v = (s[k].double() for k in ("grad", "param", "m", "v"))
    if c["state"] == 8:
        m = m * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (v * s["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g ** 2
    m_hat, v_hat = m / (1 - h["beta1"] ** t), v / (1 - h["beta2"] ** t)
    p = p - h["lr"] * (m_hat / (v_hat.sqrt() + h["eps"]) + h["weight_decay"] * p)
    out = {"param": p, "m": m, "v": v}
    if c["copy"]:
        out["copy"] = p
    if c["state"] == 8:
        out["m"] = out["v"] = None
        for k, x in (("m", m.abs()), ("v", v.sqrt())):
            top = x.view(-1, BLOCK).amax(1)
            out[k + "_scale"] = torch.where(top > 0, top / E4M3_MAX, torch.ones_like(top))
    return out
