"""The gated projections and their gradient against the oracle, within the bounds that their roundings give."""
import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2408_06995_amd import binding as B
from gpu_util import DEV
from test_gpu_blocks import E4M3, TYPES, host, nan, quantize, room, rows, within

pytestmark = pytest.mark.gpu

ACTS = {"silu": B.FPQ_GATE_SILU, "gelu": B.FPQ_GATE_GELU}


class Call:
    def __init__(self, M, N, K, t, act="silu", bias=True, ld=0, seed=1):
        g = torch.Generator().manual_seed(seed + M + N + K)
        self.M, self.N, self.K, self.bf16, self.t, self.act, self.ld = M, N, K, t == "bf16", TYPES[t], act, ld
        self.x, self.gh = rows(g, M, K, self.t, ld and K + ld), rows(g, M, N, self.t, ld and N + ld)
        self.w = torch.nn.functional.pad((torch.randn(2 * N, K, generator=g) * K ** -0.5), (0, ld), value=float("nan")).to(self.t).to(DEV)[:, :K]
        self.bias = torch.randn(2 * N, generator=g).to(DEV) if bias else None

    def forward(self, keep=None):
        """h, what is kept, its scales."""
        h = nan(self.M, self.N + self.ld, t=self.t)
        pre, scales = None, None
        if keep == "type":
            pre = nan(self.M, 2 * self.N, t=self.t)
        elif keep == "blocks":
            n = 2 * blocks.padded(self.N)
            pre, scales = (torch.full((self.M, k), 0xee, dtype=torch.uint8, device=DEV) for k in (n, n // 32))
        B.fpq_gated(self.x, self.w, self.bias, ACTS[self.act], h[:, :self.N], pre, scales, room(B.fpq_gated_workspace_size(self.M, self.N, self.K, int(self.bf16))))
        assert h[:, self.N:].isnan().all()
        return h[:, :self.N], pre, scales

    def backward(self, pre, scales, x=None, x_scales=None, gx=True, gw=True, gb=True):
        out = (nan(self.M, self.K + self.ld, t=self.t)[:, :self.K] if gx else None, nan(2 * self.N, self.K + self.ld, t=self.t)[:, :self.K] if gw else None,
               nan(2 * self.N) if gb else None)
        B.fpq_gated_backward(self.x if x is None else x, x_scales, self.w, pre, scales, ACTS[self.act], self.gh, *out,
                             room(B.fpq_gated_backward_workspace_size(self.M, self.N, self.K, int(self.bf16))))
        return out

    def kept_values(self, pre, scales):
        """a and g as they were kept, in 64 bits."""
        if scales is None:
            return host(pre[:, :self.N]), host(pre[:, self.N:])
        c, s = pre.cpu().numpy(), scales.cpu().numpy()
        half, n = c.shape[1] // 2, s.shape[1] // 2
        return blocks.block_values(c[:, :half], s[:, :n], 8, self.N), blocks.block_values(c[:, half:], s[:, n:], 8, self.N)

    def check_kept(self, pre, scales, want, off):
        for i, (got, w, o) in enumerate(zip(self.kept_values(pre, scales), want, off)):
            if scales is None:
                bad = ~(np.abs(got - w) <= o + blocks.rounding(self.bf16) * (np.abs(w) + o) + 2.0 ** -126)
            else:
                s = scales.cpu().numpy()
                s = 2.0 ** (s[:, :s.shape[1] // 2] if i == 0 else s[:, s.shape[1] // 2:]).astype(float) * 2.0 ** -127
                top, slack = np.abs(blocks._in_blocks(w)).max(2), blocks._in_blocks(o).max(2)
                assert np.all(top - slack <= 448 * s) and np.all((224 * s <= top + slack) | ((top <= slack) & (s == 1)))
                unit = np.repeat(s, 32, 1)[:, :self.N]
                bad = ~(np.abs(got - w) <= np.maximum(2.0 ** -4 * (np.abs(w) + o), 2.0 ** -10 * unit) + o * (1 + 2.0 ** -20))
                c = pre.cpu().numpy().reshape(self.M, 2, -1)
                assert not c[:, :, self.N:].any()
            assert not bad.any(), "kept: %d of %d outside" % (bad.sum(), bad.size)

    def check(self, keep="type", kept_x=False):
        bias = None if self.bias is None else host(self.bias)
        x, w = host(self.x), host(self.w)
        h, pre, scales = self.forward(keep)
        want, off, ag, d_ag = blocks.gated(x, w, bias, self.act, self.bf16)
        within("h", h, want, off)
        self.check_kept(pre, scales, ag, d_ag)
        bare = self.forward(None)[0]
        assert torch.equal(bare, h)
        xq, xs = quantize(self.x, E4M3) if kept_x else (None, None)
        xv = blocks.block_values(xq.cpu().numpy(), xs.cpu().numpy(), 8, self.K) if kept_x else x
        gx, gw, gb = self.backward(pre, scales, xq, xs)
        a, g = self.kept_values(pre, scales)
        (wx, ox), (ww, ow), (wb, ob) = blocks.gated_backward(xv, w, a, g, self.act, host(self.gh), self.bf16)
        within("grad_x", gx, wx, ox)
        within("grad_w", gw, ww, ow)
        within("grad_bias", gb, wb, ob)
        return pre, scales, gx, gw, gb


@pytest.mark.parametrize("keep", ["type", "blocks"])
@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 320, 64), (2, 33, 40), (16, 1280, 320), (17, 64, 1288), (31, 77, 328), (50, 96, 200), (33, 130, 257), (64, 32, 64), (65, 100, 72), (300, 480, 320), (129, 257, 1000),
                                   (1500, 20, 24)])
def test_sizes(M, N, K, t, keep):
    print(M, N, K, t, keep, flush=True)
    Call(M, N, K, t, "silu" if (M + N) % 2 else "gelu").check(keep)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_activations_bias_and_blocks_of_x(t, act):
    Call(70, 96, 160, t, act, bias=False).check("type")
    Call(70, 96, 160, t, act).check("blocks", kept_x=True)
    Call(31, 61, 77, t, act).check("type", kept_x=True)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("ld", [8, 3])
def test_strided_rows(ld, t):
    Call(130, 136, 72, t, "silu", ld=ld).check("type")
    Call(7, 61, 131, t, "gelu", ld=ld).check("blocks")


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_large_tiles(t):
    Call(3600, 1800, 72, t, "gelu").check("blocks")      # many tiles
    Call(40, 3000, 1000, t, "silu").check("type")        # parts along k


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gates_far_from_zero(act):
    """Gates up to +-200: nothing overflows, the tails are 0 and the gate itself."""
    M, N, K = 40, 32, 8
    c = Call(M, N, K, "fp32", act)
    c.bias = torch.cat([torch.ones(N), torch.linspace(-200, 200, N)]).to(DEV)
    pre = c.check("type")[0]
    assert pre[:, N:].abs().max() > 190


def test_each_gradient_alone_and_no_rows():
    c = Call(70, 48, 96, "bf16")
    pre, scales, gx, gw, gb = c.check("blocks")
    assert torch.equal(c.backward(pre, scales, gw=False, gb=False)[0], gx)
    assert torch.equal(c.backward(pre, scales, gx=False, gb=False)[1], gw)
    assert torch.equal(c.backward(pre, scales, gx=False, gw=False)[2], gb)
    for t in ("fp32", "bf16"):
        e = Call(0, 48, 96, t)
        h, pre, _ = e.forward("type")
        _, gw, gb = e.backward(pre, None)
        assert h.shape == (0, 48) and not gw.any() and not gb.any()


def test_rows_do_not_depend_on_each_other():
    c = Call(16, 128, 320, "bf16")
    h = c.forward()[0]
    c.x[3, 7] = float("nan")
    z = c.forward()[0]
    keep = [m for m in range(16) if m != 3]
    assert torch.equal(h[keep], z[keep]) and z[3].isnan().all()
    one = Call(16, 128, 320, "bf16")
    one.x, one.M = one.x[4:5], 1
    assert torch.equal(one.forward()[0], h[4:5])
