"""numpy oracle, in 64 bits, of the operators around a transformer block's projections: blocks of codes with a power of two as their
scale, gradients of linear layers, gated projections, root-mean-square norm on the residual stream.

Next to a result, `bounds` give how far a computation in 32-bit sums may be from it: every rounding it makes, times what that rounding
scales."""
import math

import numpy as np

from .adapt import U16, U32

TOP = {8: (8, 0.875), 4: (2, 0.75)}               # largest value: m 2^(e + 1)
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def padded(n):
    return -(-n // 32) * 32


def e4m3_values():
    """The values of the 127 codes without sign that are numbers."""
    c = np.arange(127)
    p, f = c >> 3, c & 7
    return np.where(p == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * 2.0 ** (p - 7.0))


def _in_blocks(x):
    M, K = x.shape
    b = np.zeros((M, padded(K)))
    b[:, :K] = x
    return b.reshape(M, -1, 32)


def block_scales(x, bits):
    """Exponents, biased by 127, of the least power of two with which a block is in range; 255 for blocks that are not finite."""
    b = _in_blocks(np.asarray(x, np.float64))
    with np.errstate(invalid="ignore"):
        top = np.abs(b).max(2)
    exp, m = TOP[bits]
    fine = np.isfinite(top)
    f, e = np.frexp(np.where(fine, top, 0.0))
    s = np.where(f == 0, 0, np.maximum(e - 1 - exp + (f > m), -126)) + 127
    return np.where(fine, s, 255).astype(np.uint8)


def _grid(bits):
    return e4m3_values() if bits == 8 else E2M1


def block_quantize(x, bits, mask=None):
    """codes [M, padded(K)], one per element, and scales; NaN blocks have unspecified codes."""
    x = np.asarray(x, np.float64)
    s = block_scales(x, bits)
    b = _in_blocks(x) * 2.0 ** (127.0 - np.where(s == 255, 127, s).astype(np.float64))[:, :, None]
    b = np.where(np.isfinite(b), b, 0.0)
    grid = _grid(bits)
    a = np.abs(b)
    hi = np.clip(np.searchsorted(grid, a, side="left"), 0, len(grid) - 1)      # first value >= a
    lo = np.maximum(hi - 1, 0)
    if mask is None:
        up, down = grid[hi] - a, a - grid[lo]
        code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
        neg = np.signbit(b)
    else:
        # Eq. (12): down to a multiple of the step of the value's own binade, one step more where the mask says so, within the range
        h = np.zeros(b.shape).reshape(len(x), -1)
        h[:, :x.shape[1]] = np.asarray(mask) != 0
        s = block_scales(x, bits)
        step = 2.0 ** (np.maximum(np.frexp(a)[1] - 1.0, 0) - 1)
        v = np.clip((np.floor(b / step) + h.reshape(b.shape)) * step, -6, 6)
        code, neg = np.searchsorted(grid, np.abs(v)), (v < 0) | ((v == 0) & np.signbit(b))
    out = (code | (neg.astype(np.int64) << (7 if bits == 8 else 3))).astype(np.uint8).reshape(len(x), -1)
    out[:, x.shape[1]:] = 0
    return out, s


def block_values(codes, scales, bits, K):
    """[M, K] of codes one per element."""
    grid = np.append(_grid(bits), np.nan) if bits == 8 else E2M1
    top = 7 if bits == 8 else 3
    v = grid[codes & ((1 << top) - 1)] * np.where(codes >> top, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (np.where(scales == 255, 127, scales).astype(np.float64) - 127))
    return (v.reshape(len(codes), -1, 32) * s[:, :, None]).reshape(len(codes), -1)[:, :K]


def nibbles(codes):
    """Codes one per element -> two per byte."""
    return codes[:, 0::2] | codes[:, 1::2] << 4


def unpack(packed):
    return np.stack([packed & 15, packed >> 4], 2).reshape(len(packed), -1)


# ------------------------------------------------------------------------------------------------ products

def product(a, b, r, extra=0.0):
    """a [M, K] times b [N, K] transposed and its bound: sums of fp32 order, operands off by `extra` [M, K] already, the result's own
    rounding r."""
    y = a @ b.T
    mass = np.abs(a) @ np.abs(b).T
    off = (a.shape[1] + 16) * U32 * mass
    if np.ndim(extra):
        off = off + (extra @ np.abs(b).T) * (1 + 2.0 ** -10)
    return y, off + r * (np.abs(y) + off) + 2.0 ** -126


def rounding(bf16):
    return U16 if bf16 else U32


def linear_backward(x, w, gy, bf16):
    """(grad_x, grad_w, grad_bias), each with its bound."""
    r = rounding(bf16)
    gb = gy.sum(0)
    return product(gy, w.T, r), product(gy.T, x.T, r), (gb, (len(gy) + 2) * U32 * np.abs(gy).sum(0) + 2.0 ** -126)


def block_linear(x, w, bias, bf16):
    y, off = product(x, w, rounding(bf16))
    if bias is not None:
        y = y + bias
        off = off + (rounding(bf16) + U32) * (np.abs(bias) + np.abs(y))
    return y, off


# ------------------------------------------------------------------------------------------------ gated projections

_erf = np.vectorize(math.erf, otypes=[np.float64])


def gate(g, act):
    """act(g), its derivative, and how far the kernels' formulas may be from either."""
    big = np.abs(g)
    if act == "silu":
        e = np.exp(-big)
        z = np.where(g >= 0, 1 / (1 + e), e / (1 + e))
        dz = (4 + big) * 2.0 ** -23 * z
        # The slope z s, s = 1 + g q, q = 1 - z.  z = 1 / (1 + e^-g) is off by the exponential's (1 + |g|) 2^-23 as far as it counts in the sum, by the sum's
        # 2^-24 and the reciprocal's 2^-23; q by that and a rounding, s by |g| times as much and a rounding.  (A sigmoid below the smallest normal
        # number, 2^-126, may be zero.)
        q = np.where(g >= 0, e / (1 + e), 1 / (1 + e))
        s = 1 + g * q
        d_z = z * (q * (1 + big) + 2) * 2.0 ** -23 + 2.0 ** -126
        d_s = big * (d_z + U32 * q) + U32 * np.abs(s)
        return g * z, z * s, big * (dz + U32 * z + 2.0 ** -126), z * d_s + d_z * (np.abs(s) + d_s) + 2 * U32 * np.abs(z * s)
    z = 0.5 * (1 + _erf(g * 0.5 ** 0.5))
    z = np.where(g < -1, 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-g * 0.5 ** 0.5), z)
    phi = np.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5
    return g * z, z + g * phi, 4e-7 * big + U32 * big, np.full_like(g, 6e-7) + 2 * U32


def gated(x, w, bias, act, bf16):
    """h and its bound, a and g (64 bits) and theirs."""
    N = len(w) // 2
    pre, off = product(x, w, 0.0)
    if bias is not None:
        pre = pre + bias
        off = off + U32 * (np.abs(pre) + np.abs(bias))
    a, g, da, dg = pre[:, :N], pre[:, N:], off[:, :N], off[:, N:]
    f, _, df, _ = gate(g, act)
    h = a * f
    off_h = (np.abs(a) + da) * (df + 1.13 * dg) + da * np.abs(f) + 2 * U32 * np.abs(h)
    return h, off_h + rounding(bf16) * (np.abs(h) + off_h) + 2.0 ** -126, (a, g), (da, dg)


def gated_backward(x, w, a, g, act, gh, bf16):
    """(grad_x, grad_w, grad_bias) from a and g as they were kept, each with its bound."""
    r = rounding(bf16)
    f, slope, df, ds = gate(g, act)
    d = np.concatenate([gh * f, gh * a * slope], 1)
    off = np.concatenate([np.abs(gh) * df, np.abs(gh * a) * ds], 1) + 4 * U32 * np.abs(d)
    gb = d.sum(0)
    off_gb = off.sum(0) + (len(x) + 2) * U32 * (np.abs(d) + off).sum(0) + 2.0 ** -126
    # (of two bf16 parts or three; one below the smallest normal number may be zero: what is left out is below 2^-125)
    as_operand = off + (U16 ** 2 if bf16 else 2 * U32) * (np.abs(d) + off) + 2.0 ** -125
    return product(d, w.T, r, as_operand), product(d.T, x.T, r, as_operand.T), (gb, off_gb)


def gated_spread(x, w, a, g, act, gh):
    """How far bf16 grad_x and grad_w are off ahead of their own rounding: a standard deviation per element, da and dg as operands of 16 bits,
    whose roundings are independent and uniform, and bounds for the activation and for sums in 32 bits."""
    f, slope, df, ds = gate(g, act)
    d = np.concatenate([gh * f, gh * a * slope], 1)
    own = np.concatenate([np.abs(gh) * df, np.abs(gh * a) * ds], 1) + (U16 ** 2 * 3.0 ** -0.5 + 4 * U32) * np.abs(d)
    sums = lambda p, q: np.sqrt((p[0] * p[0]) @ (q * q)) + (len(q) + 16) * U32 * (np.abs(p[1]) @ np.abs(q))
    return sums((own, d), w), sums((own.T, d.T), x)


# ------------------------------------------------------------------------------------------------ norm

def rms_norm(r, w, eps):
    """y and rstd of the stream r, with bounds ahead of a result's own rounding."""
    K = r.shape[1]
    rstd = 1 / np.sqrt((r * r).mean(1, keepdims=True) + eps)
    rel = (K / 2 + 8) * U32
    y = r * rstd * w
    return y, np.abs(y) * (rel + 4 * U32), rstd[:, 0], rstd[:, 0] * rel


def rms_norm_backward(r, w, rstd, gy, gs):
    """(grad_x, grad_w) from rstd as it was kept, with bounds ahead of a result's own rounding."""
    K = r.shape[1]
    s = rstd[:, None]
    g = gy * w
    c = (g * r).mean(1, keepdims=True) * s * s
    gx = s * (g - r * c) + gs
    mass = np.abs(g * r).mean(1, keepdims=True) * s * s
    off = s * (4 * U32 * np.abs(g) + np.abs(r) * (K + 12) * U32 * mass) + 4 * U32 * (np.abs(gx) + np.abs(gs) + s * np.abs(g) + s * np.abs(r * c))
    gw = (gy * r * s).sum(0)
    return gx, off, gw, (len(r) + 8) * U32 * np.abs(gy * r * s).sum(0)
