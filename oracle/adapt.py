"""numpy oracle, in 64 bits, of the operators for adapting a quantized model: attention and its gradient, low-rank adapters and
theirs, AdamW.

Next to a result, `bounds` functions give how far a computation in 32-bit sums may be from it: every rounding it makes, times what
that rounding scales."""
import numpy as np

U32 = 2.0 ** -24              # half a unit in the last place of an fp32 number near 1
U16 = 2.0 ** -8               # and of a bf16 number, which has 8 significant bits


def keys_of(lens, b, kv_len):
    return kv_len if lens is None else int(min(max(int(lens[b]), 0), kv_len))


def visible(q_len, n, causal):
    """[q_len, n]: which keys a query sees."""
    i, j = np.arange(q_len)[:, None], np.arange(n)[None, :]
    return (j <= i + n - q_len) if causal else np.ones((q_len, n), bool)


def _head(q, k, v, b, x, group, n):
    f = np.float64
    return q[b, :, x].astype(f), k[b, :n, x // group].astype(f), v[b, :n, x // group].astype(f)


def _probabilities(Q, K, scale, causal):
    """p and lse of one head; rows that see nothing: zeros and -infinity."""
    see = visible(len(Q), len(K), causal)
    s = np.where(see, scale * (Q @ K.T), -np.inf)
    top = s.max(1, initial=-np.inf, keepdims=True)
    some = np.isfinite(top)
    e = np.where(see, np.exp(s - np.where(some, top, 0.0)), 0.0)
    total = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = np.where(some, top + np.log(total), -np.inf)[:, 0]
    return np.where(some, e / np.where(total > 0, total, 1.0), 0.0), lse


def attention(q, k, v, scale, causal=False, lens=None):
    """o, lse of [B, L, H, D] arrays."""
    B, Lq, Hq, D = q.shape
    o, lse = np.zeros(q.shape), np.full((B, Hq, Lq), -np.inf)
    for b in range(B):
        n = keys_of(lens, b, k.shape[1])
        for x in range(Hq):
            Q, K, V = _head(q, k, v, b, x, Hq // k.shape[2], n)
            p, lse[b, x] = _probabilities(Q, K, scale, causal)
            o[b, :, x] = p @ V
    return o, lse


def attention_backward(q, k, v, go, scale, causal=False, lens=None):
    gq, gk, gv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    G = q.shape[2] // k.shape[2]
    for b in range(q.shape[0]):
        n = keys_of(lens, b, k.shape[1])
        for x in range(q.shape[2]):
            Q, K, V = _head(q, k, v, b, x, G, n)
            dO = go[b, :, x].astype(np.float64)
            p, _ = _probabilities(Q, K, scale, causal)
            dp = dO @ V.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            gq[b, :, x] = scale * (ds @ K)
            gk[b, :n, x // G] += scale * (ds.T @ Q)
            gv[b, :n, x // G] += p.T @ dO
    return gq, gk, gv


def attention_bounds(q, k, v, scale, causal, lens, bf16, go=None):
    """Bounds of |error| for o and lse (and, with go, for gq, gk, gv).

    A score's error is that of its fp32 sum, D + 16 roundings (16: the parts of a split operand and the scale) of at most
    scale sum |q k|; a probability's relative error is e^2d - 1 for scores within d, with a few roundings of its own.  Sums over
    n terms make n roundings.  With bf16 operands, p and ds are rounded once more where they are multiplied, and so are results."""
    B, Lq, Hq, D = q.shape
    G = Hq // k.shape[2]
    r = U16 if bf16 else 4 * U32                       # of p or ds as an operand, and of a result
    to, tl = np.zeros(q.shape), np.zeros((B, Hq, Lq))
    tq, tk, tv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b in range(B):
        n = keys_of(lens, b, k.shape[1])
        for x in range(Hq):
            Q, K, V = _head(q, k, v, b, x, G, n)
            p, lse = _probabilities(Q, K, scale, causal)
            see = visible(Lq, n, causal)
            mass = np.where(see, scale * (np.abs(Q) @ np.abs(K).T), 0.0).max(1, initial=0.0, keepdims=True)
            d = (D + 16) * U32 * mass + 8 * U32
            dp_rel = np.expm1(2 * d) + (n + 16) * U32  # of a normalised probability
            tl[b, x] = (d[:, 0] + (n + 16) * U32) + 2 * U32 * np.abs(np.where(np.isfinite(lse), lse, 0.0))
            pv = p @ np.abs(V)
            to[b, :, x] = pv * (dp_rel + r + (n + 8) * U32) * (1 + r) + r * np.abs(p @ V)
            if go is None:
                continue
            dO = go[b, :, x].astype(np.float64)
            A = np.abs(dO) @ np.abs(V).T
            dp = dO @ V.T
            delta = (p * dp).sum(1, keepdims=True)
            d_delta = (np.abs(dO) * to[b, :, x]).sum(1, keepdims=True) + (D + 8) * U32 * (np.abs(dO) * pv).sum(1, keepdims=True)
            ds = p * (dp - delta)
            d_ds = p * ((D + 16) * U32 * A + d_delta) * (1 + dp_rel) + np.abs(ds) * (dp_rel + r + 4 * U32)
            m_ds = np.abs(ds) + d_ds
            tq[b, :, x] = scale * (d_ds @ np.abs(K) + (n + 8) * U32 * (m_ds @ np.abs(K)))
            tk[b, :n, x // G] += scale * (d_ds.T @ np.abs(Q) + (G * Lq + 8) * U32 * (m_ds.T @ np.abs(Q)))
            tv[b, :n, x // G] += (p * (dp_rel + r + (G * Lq + 8) * U32)).T @ np.abs(dO) * (1 + r)
    if go is None:
        return to, tl
    gq, gk, gv = attention_backward(q, k, v, go, scale, causal, lens)
    return to, tl, tq + r * np.abs(gq), tk + r * np.abs(gk), tv + r * np.abs(gv)


def attention_spread(q, k, v, scale, causal, lens, go=None):
    """How far results of bf16 attention are off ahead of their own rounding, for o (and, with go, for gq, gk, gv): a standard deviation per
    element, roundings taken as independent and uniform where they are of many values, and as a bound where one is shared or made in
    32 bits.

    Probabilities and their gradients as operands keep 16 bits, u = U16^2; delta = do . o takes o as it was rounded to bf16."""
    B, Lq, Hq, D = q.shape
    G, third = Hq // k.shape[2], 3.0 ** -0.5
    so, sq = np.zeros(q.shape), np.zeros(q.shape)
    k2, k1, v2, v1 = (np.zeros(k.shape) for _ in range(4))             # squares of what is independent, and what adds up
    for b in range(B):
        n = keys_of(lens, b, k.shape[1])
        for x in range(Hq):
            Q, K, V = _head(q, k, v, b, x, G, n)
            p, lse = _probabilities(Q, K, scale, causal)
            mass = np.where(visible(Lq, n, causal), scale * (np.abs(Q) @ np.abs(K).T), 0.0).max(1, initial=0.0, keepdims=True)
            # a probability's own relative error, and what it shares with its row (the sum, the log-sum)
            s = U16 ** 2 * third + (D + 16) * U32 * mass + 8 * U32
            row = s + (n + 16) * U32 + 2 * U32 * np.abs(np.where(np.isfinite(lse), lse, 0.0))[:, None]
            o = p @ V
            so[b, :, x] = s * np.sqrt((p * p) @ (V * V)) + row * np.abs(o) + (n + 8) * U32 * (p @ np.abs(V))
            if go is None:
                continue
            dO = go[b, :, x].astype(np.float64)
            dp = dO @ V.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            d_delta = np.sqrt((dO ** 2 * ((U16 * third * o) ** 2 + so[b, :, x] ** 2)).sum(1, keepdims=True)) + (D + 8) * U32 * (np.abs(dO) * np.abs(o)).sum(1, keepdims=True)
            own = np.abs(ds) * (s + row) + p * (D + 16) * U32 * (np.abs(dO) @ np.abs(V).T)
            sq[b, :, x] = scale * (np.sqrt((own * own) @ (K * K)) + d_delta * np.abs(p @ K) + row * np.abs(ds @ K) + (n + 8) * U32 * (np.abs(ds) @ np.abs(K)))
            k2[b, :n, x // G] += scale ** 2 * ((own * own + (p * d_delta) ** 2).T @ (Q * Q))
            k1[b, :n, x // G] += scale * (G * Lq + 8) * U32 * (np.abs(ds).T @ np.abs(Q))
            v2[b, :n, x // G] += ((p * (s + row)) ** 2).T @ (dO * dO)
            v1[b, :n, x // G] += (G * Lq + 8) * U32 * (p.T @ np.abs(dO))
    return (so,) if go is None else (so, sq, np.sqrt(k2) + k1, np.sqrt(v2) + v1)


def bf16(x):
    """Rounded to bf16, to nearest even (finite values within its range)."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32).astype(np.float64)


def off_in_norm(got, want, spread):
    """The squared distance of bf16 results `got` from `want` rounded to bf16, over the largest that `spread` gives it.

    A value that is off by e before it is rounded comes out one unit in the last place, w, beside the right one with a probability of
    |e| / w: its square is w |e| + e^2 on average, and its variance at most w^3 |e|.  Four of its standard deviations, and half as much
    again on the average for errors that share a rounding."""
    w = np.where(want == 0, 0.0, 2.0 ** (np.floor(np.log2(np.where(want == 0, 1.0, np.abs(want)))) - 7))
    most = 1.5 * (spread * w + spread ** 2).sum() + 4 * np.sqrt((spread * w ** 3).sum())
    return ((got - bf16(want)) ** 2).sum() / most


# ------------------------------------------------------------------------------------------------ AdamW

BLOCK, E4M3_MAX = 256, 448.0


def e4m3_values():
    """Value of every code of the format (4, 3, 7, 448); the two codes without one are NaN."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v).astype(np.float32)


def e4m3_codes(x):
    """Codes of fp32 values of magnitude at most 448, to nearest, ties to the even code."""
    grid = e4m3_values()[:127].astype(np.float64)
    a = np.abs(x.astype(np.float64))
    hi = np.minimum(np.searchsorted(grid, a), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def state_codes(x, root):
    """8-bit codes and scales of a flat fp32 state (a root of v: a positive value gets no code 0)."""
    n = len(x)
    b = np.zeros(-(-n // BLOCK) * BLOCK, np.float32)
    b[:n] = x
    b = b.reshape(-1, BLOCK)
    top = np.abs(b).max(1)
    scale = np.where(top == 0, np.float32(1), np.maximum(top * np.float32(np.float32(1) / np.float32(E4M3_MAX)), np.float32(2.0 ** -126))).astype(np.float32)
    y = np.clip(b * (np.float32(1) / scale)[:, None], np.float32(-E4M3_MAX), np.float32(E4M3_MAX))
    if root:
        y = np.where(b > 0, np.maximum(y, np.float32(2.0 ** -9)), y)
    return e4m3_codes(y.reshape(-1)[:n]), scale


def state_values(codes, scale):
    return (e4m3_values()[codes] * np.repeat(scale, BLOCK)[:len(codes)]).astype(np.float32)


def adamw(param, grad, m, v, lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0):
    """param, m, v after one step, in the precision of the arrays (all of one type), every operation rounded by itself."""
    t = param.dtype.type
    g = grad * t(grad_scale)
    m = m * t(beta1) + g * t(1 - beta1)
    v = v * t(beta2) + g * t(1 - beta2) * g
    by = m / (np.sqrt(v) * t((1 - beta2 ** step) ** -0.5) + t(eps))
    return param * t(1 - lr * weight_decay) - by * t(lr / (1 - beta1 ** step)), m, v


# ------------------------------------------------------------------------------------------------ adapters

def requests_of(row_start, adapter, M, adapters):
    """(rows, adapter) of the requests that have one."""
    for r, i in enumerate(adapter):
        lo, hi = (int(min(max(v, 0), M)) for v in row_start[r:r + 2])
        if 0 <= i < adapters and lo < hi:
            yield slice(lo, hi), int(i)


def adapter_apply(x, a, b, scaling, row_start, adapter, base):
    """y, t."""
    y, t = base.astype(np.float64).copy(), np.zeros((len(x), a.shape[1]))
    for rows, i in requests_of(row_start, adapter, len(x), len(a)):
        t[rows] = x[rows] @ a[i].T
        y[rows] += scaling[i] * (t[rows] @ b[i].T)
    return y, t


def adapter_backward(x, a, b, scaling, row_start, adapter, gy, gx_base):
    """gx, ga, gb."""
    gx, ga, gb = gx_base.astype(np.float64).copy(), np.zeros(a.shape), np.zeros(b.shape)
    for rows, i in requests_of(row_start, adapter, len(x), len(a)):
        t, dt = x[rows] @ a[i].T, scaling[i] * (gy[rows] @ b[i])
        gx[rows] += dt @ a[i]
        ga[i] += dt.T @ x[rows]
        gb[i] += scaling[i] * (gy[rows].T @ t)
    return gx, ga, gb


def adapter_bounds(x, a, b, scaling, row_start, adapter, base, bf16, gy=None, gx_base=None):
    """Bounds of |error| for y and t (and, with gy, for gx, ga, gb): a sum over n terms makes n + 16 roundings (16: the parts of split
    operands, the scale, the sum of parts) of at most the sum of its terms' magnitudes, on top of what its operands are off."""
    u = lambda n: (n + 16) * U32
    r = U16 if bf16 else U32
    M, (_, R, K), N = len(x), a.shape, b.shape[1]
    t_off, y_off = np.zeros((M, R)), np.zeros((M, N))
    A, B, X = np.abs(a), np.abs(b), np.abs(x)
    y, _ = adapter_apply(x, a, b, scaling, row_start, adapter, base)
    out = []
    for rows, i in requests_of(row_start, adapter, M, len(a)):
        mass = X[rows] @ A[i].T
        t_off[rows] = u(K) * mass
        y_off[rows] = scaling[i] * ((t_off[rows] + u(R) * mass) @ B[i].T)
    y_off += U32 * (np.abs(base) + np.abs(y)) + r * (np.abs(y) + y_off)
    if gy is None:
        return y_off, t_off
    gx_off, ga_off, gb_off = np.zeros((M, K)), np.zeros(a.shape), np.zeros(b.shape)
    G = np.abs(gy)
    gx, _, _ = adapter_backward(x, a, b, scaling, row_start, adapter, gy, gx_base)
    for rows, i in requests_of(row_start, adapter, M, len(a)):
        mass_t, mass_d = X[rows] @ A[i].T, scaling[i] * (G[rows] @ B[i])
        d_off = u(N) * mass_d
        gx_off[rows] = (d_off + u(R) * mass_d) @ A[i]
        ga_off[i] += (d_off + u(M) * mass_d).T @ X[rows]
        gb_off[i] += scaling[i] * (G[rows].T @ (t_off[rows] + u(M) * mass_t))
    gx_off += U32 * (np.abs(gx_base) + np.abs(gx)) + r * (np.abs(gx) + gx_off)
    return y_off, t_off, gx_off, ga_off, gb_off
