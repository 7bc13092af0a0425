"""AdamW over many tensors: fp32 results within the roundings of the formula in 64 bits, and bit for bit what the formula gives when
it is evaluated in fp32, operation by operation; 8-bit codes and scales equal."""
import numpy as np
import pytest
import torch

from oracle import adapt
from paper_2408_06995_amd import binding as B
from gpu_util import DEV

pytestmark = pytest.mark.gpu

U = adapt.U32
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
HYPER = (3e-3, 0.9, 0.999, 1e-8, 0.05)


class Tensor:
    """One tensor of a set, on the device and as host arrays."""

    def __init__(self, n, bits, param, grad, copy, seed, offset=0, state_type=torch.uint8):
        rng = np.random.default_rng(seed)
        self.n, self.bits, self.keep = n, bits, []
        p, g, m = (rng.standard_normal(n).astype(np.float32) * s for s in (np.float32(0.1), np.float32(1e-2), np.float32(1e-3)))
        g *= np.exp2(rng.integers(-12, 4, n)).astype(np.float32)
        v = (m * m + (rng.standard_normal(n) * 1e-3).astype(np.float32) ** 2).astype(np.float32)
        self.param, self.grad = self.place(p, TYPES[param], offset), self.place(g, TYPES[grad], offset)
        self.copy = self.place(np.zeros(n, np.float32), torch.bfloat16, offset) if copy else None
        self.scales = [None, None]
        if bits == 32:
            self.m, self.v = self.place(m, torch.float32, offset), self.place(v, torch.float32, offset)
            self.host_m, self.host_v = m, v
        else:
            (mc, ms), (vc, vs) = adapt.state_codes(m, False), adapt.state_codes(np.sqrt(v), True)
            self.m, self.v = (self.place(c, torch.uint8, offset) for c in (mc, vc))
            if state_type != torch.uint8:
                self.m, self.v = self.m.view(state_type), self.v.view(state_type)
            self.scales = [torch.from_numpy(s).to(DEV) for s in (ms, vs)]
            self.host_m, self.host_v = adapt.state_values(mc, ms), adapt.state_values(vc, vs) ** 2
        self.host_p, self.host_g = (x.float().cpu().numpy() for x in (self.param, self.grad))

    def place(self, a, t, offset):
        """On the device, `offset` elements into a buffer whose other elements must keep their values."""
        buf = torch.full((offset + len(a) + 5,), 7, device=DEV, dtype=t)
        buf[offset:offset + len(a)] = torch.from_numpy(a).to(DEV).to(t)
        self.keep.append((buf, offset, len(a)))
        return buf[offset:offset + len(a)]

    def item(self):
        return (self.param, self.grad, self.m, self.v, *self.scales, self.copy)

    def check(self, step, grad_scale=1.0):
        lr, b1, b2, eps, wd = HYPER
        with np.errstate(all="ignore"):
            p, m, v = adapt.adamw(self.host_p, self.host_g, self.host_m, self.host_v, *HYPER, step, np.float32(grad_scale))
            P, M, V = adapt.adamw(*(x.astype(np.float64) for x in (self.host_p, self.host_g, self.host_m, self.host_v)), *HYPER, step,
                                  float(np.float32(grad_scale)))
        # a product and the sum, with constants rounded once: 3 U of each term; v: one product more
        size_m = np.abs(self.host_m.astype(np.float64)) * b1 + np.abs(self.host_g.astype(np.float64) * grad_scale) * (1 - b1)
        tm, tv = 5 * U * size_m + 1e-44, 8 * U * V + 1e-44
        denom = np.sqrt(V) * (1 - b2 ** step) ** -0.5 + eps
        size = lr / (1 - b1 ** step)
        tp = 3 * U * np.abs(self.host_p) + size * (tm / denom + 16 * U * np.abs(M) / denom) + U * np.abs(P)
        assert np.all(np.abs(p - P) <= tp) and np.all(np.abs(m - M) <= tm) and np.all(np.abs(v - V) <= tv), "the oracle in 32 bits"
        want = torch.from_numpy(p).to(self.param.dtype)
        assert torch.equal(self.param.cpu(), want), "param"
        if self.copy is not None:
            assert torch.equal(self.copy.cpu(), torch.from_numpy(p).bfloat16()), "copy"
        if self.bits == 32:
            assert np.array_equal(self.m.cpu().numpy(), m) and np.array_equal(self.v.cpu().numpy(), v), "states"
            self.host_m, self.host_v = m, v
        else:
            for got, scale, x, root in ((self.m, self.scales[0], m, False), (self.v, self.scales[1], np.sqrt(v), True)):
                codes, s = adapt.state_codes(x, root)
                assert np.array_equal(scale.cpu().numpy(), s), "scales"
                assert np.array_equal(got.view(torch.uint8).cpu().numpy(), codes), "codes"
            self.host_m, self.host_v = (adapt.state_values(t.view(torch.uint8).cpu().numpy(), s.cpu().numpy()) for t, s in
                                        ((self.m, self.scales[0]), (self.v, self.scales[1])))
            self.host_v = (self.host_v * self.host_v).astype(np.float32)
        self.host_p = self.param.float().cpu().numpy()
        for buf, first, n in self.keep:
            rest = torch.cat([buf[:first], buf[first + n:]]).float()
            assert torch.all(rest == 7), "outside the tensor"


def plan_of(tensors):
    arr = B.adamw_tensors([t.item() for t in tensors])
    plan = torch.empty(B.fpq_adamw_plan_size(arr), dtype=torch.uint8, device=DEV)
    return plan, B.fpq_adamw_plan(arr, plan)


SIZES = [1, 3, 4, 255, 256, 257, 1023, 2047, 2048, 2049, 5000, 100000]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,copy", [("fp32", "fp32", True), ("fp32", "bf16", False), ("bf16", "fp32", False), ("bf16", "bf16", True)])
def test_steps(bits, param, grad, copy):
    tensors = [Tensor(n, bits, param, grad, copy, n + bits, offset=0 if n % 2 else n % 3) for n in SIZES]
    plan, pieces = plan_of(tensors)
    for step in (1, 2, 50):
        B.fpq_adamw_step(plan, pieces, *HYPER, step)
        for t in tensors:
            t.check(step)


def test_mixed_set_of_many_and_a_scale_of_the_gradient():
    rng = np.random.default_rng(9)
    tensors = [Tensor(int(rng.integers(1, 6000)), [32, 8][i % 2], ["fp32", "bf16"][i // 2 % 2], ["fp32", "bf16"][i // 4 % 2], i % 3 == 0, i,
                      offset=i % 5, state_type=[torch.uint8, torch.float8_e4m3fn][i % 4 // 2]) for i in range(75)]
    plan, pieces = plan_of(tensors)
    assert pieces == sum(-(-t.n // 2048) for t in tensors)
    scale = torch.tensor([0.37], device=DEV)
    B.fpq_adamw_step(plan, pieces, *HYPER, 3, scale)
    for t in tensors:
        t.check(3, float(scale.item()))


def test_empty_tensors_and_an_empty_set():
    a, b = Tensor(0, 32, "fp32", "fp32", False, 1), Tensor(300, 8, "fp32", "fp32", False, 2)
    plan, pieces = plan_of([a, b, a])
    assert pieces == 1
    B.fpq_adamw_step(plan, pieces, *HYPER, 1)
    b.check(1)
    empty = B.adamw_tensors([])
    assert B.fpq_adamw_plan(empty, plan) == 0
    B.fpq_adamw_step(plan, 0, *HYPER, 1)


@pytest.mark.parametrize("bits", [32, 8])
def test_states_of_zero_tiny_and_large_gradients(bits):
    t = Tensor(1024, bits, "fp32", "fp32", False, 4)
    g = np.zeros(1024, np.float32)
    g[256:512] = np.float32(1e-30)                    # squares to zero: the update divides by eps alone
    g[512:768] = np.float32(3e18)
    g[700] = np.float32(1e-44)
    t.grad.copy_(torch.from_numpy(g))
    t.host_g = g
    for s in (t.m, t.v):
        s.zero_()
    t.host_m, t.host_v = np.zeros(1024, np.float32), np.zeros(1024, np.float32)
    plan, pieces = plan_of([t])
    for step in (1, 2):
        B.fpq_adamw_step(plan, pieces, *HYPER, step)
        t.check(step)


def test_a_gradient_that_is_no_number_stays_in_its_block():
    for bad in (float("nan"), float("inf")):
        t = Tensor(1000, 8, "fp32", "fp32", False, 5)
        before = t.param.clone()
        t.grad[300] = bad
        plan, pieces = plan_of([t])
        B.fpq_adamw_step(plan, pieces, *HYPER, 1)
        p = t.param.cpu()
        assert torch.isnan(p[300]) and torch.isfinite(torch.cat([p[:300], p[301:]])).all()
        assert not torch.isfinite(t.scales[0][1]) and torch.isfinite(t.scales[0][[0, 2, 3]]).all()
        B.fpq_adamw_step(plan, pieces, *HYPER, 2)
        p = t.param.cpu()
        assert torch.isfinite(p[:256]).all() and torch.isfinite(p[512:]).all() and torch.isnan(p[256:512]).any()
        assert not torch.equal(before.cpu()[:256], p[:256])


def test_a_graph_of_steps():
    t, u = (Tensor(3000, 8, "fp32", "fp32", True, 6) for _ in range(2))
    plan, pieces = plan_of([t])
    other, _ = plan_of([u])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.fpq_adamw_step(plan, pieces, *HYPER, 5)
    for _ in range(3):
        graph.replay()
        B.fpq_adamw_step(other, pieces, *HYPER, 5)
        torch.cuda.synchronize()
        assert torch.equal(t.param, u.param) and torch.equal(t.m, u.m) and torch.equal(t.v, u.v) and torch.equal(t.copy, u.copy)
