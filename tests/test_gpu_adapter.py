"""Low-rank adapters of many requests and their gradients against the oracle in 64 bits, within the bounds that their roundings give."""
import numpy as np
import pytest
import torch

from oracle import adapt
from paper_2408_06995_amd import binding as B
from gpu_util import DEV

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
PAIRS = [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")]


def room(n):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=DEV)


def nan(*shape, t=torch.float32):
    return torch.full(shape, float("nan"), dtype=t, device=DEV)


def host(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


class Call:
    def __init__(self, M, N, K, R, starts, of, adapters, x="fp32", w="fp32", seed=1):
        g = torch.Generator().manual_seed(seed)
        t, tw = TYPES[x], TYPES[w]
        rand = lambda *s: torch.randn(*s, generator=g)
        self.x, self.base, self.gy, self.gx_base = (rand(M, n).to(t).to(DEV) for n in (K, N, N, K))
        self.a, self.b = (rand(adapters, R, K) * K ** -0.5).to(tw).to(DEV), (rand(adapters, N, R) * 0.2).to(tw).to(DEV)
        self.scaling = (torch.rand(adapters, generator=g) + 0.5).to(DEV)
        self.starts, self.of = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in (starts, of))
        self.sizes = (M, N, K, R, len(of), adapters)
        self.shared = (self.x, self.a, self.b, self.scaling, self.starts, self.of)

    def forward(self, base=True, y=None, keep_t=True):
        M, N, K, R = self.sizes[:4]
        y = nan(M, N, t=self.x.dtype) if y is None else y
        t = nan(M, R) if keep_t else None
        base = self.base if base is True else base
        B.fpq_adapter_apply(self.x, self.a, self.b, self.scaling, self.starts, self.of, base, y, t, room(B.fpq_adapter_workspace_size(*self.sizes)))
        return y, t

    def backward(self, t, base=True, gx=True):
        M, N, K, R = self.sizes[:4]
        gx = nan(M, K, t=self.x.dtype) if gx is True else gx
        ga, gb = nan(*self.a.shape), nan(*self.b.shape)
        base = self.gx_base if base is True else base
        B.fpq_adapter_backward(self.x, self.a, self.b, self.scaling, self.starts, self.of, t, self.gy, base, gx, ga, gb,
                               room(B.fpq_adapter_backward_workspace_size(*self.sizes)))
        return gx, ga, gb

    def check(self):
        y, t = self.forward()
        gx, ga, gb = self.backward(t)
        torch.cuda.synchronize()
        v = [host(z) for z in (self.x, self.a, self.b, self.scaling)] + [self.starts.cpu().numpy(), self.of.cpu().numpy()]
        base, gy, gx_base = (host(z) for z in (self.base, self.gy, self.gx_base))
        want = [*adapt.adapter_apply(*v, base), *adapt.adapter_backward(*v, gy, gx_base)]
        off = adapt.adapter_bounds(*v, base, self.x.dtype == torch.bfloat16, gy, gx_base)
        for name, got, w, o in zip(("y", "t", "gx", "ga", "gb"), (y, t, gx, ga, gb), want, off):
            err = np.abs(host(got) - w)
            bad = ~(err <= o)
            assert not bad.any(), "%s: %d of %d outside, worst %.3g of the bound" % (name, bad.sum(), bad.size, np.nanmax(err / (o + 1e-30)))
        return y, t, gx, ga, gb


RAGGED = ([0, 1, 1, 34, 66, 130, 131], [2, 0, 0, 1, -1, 2])


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("R", [1, 8, 16, 20, 32, 33, 64, 100, 128])
@pytest.mark.parametrize("N,K", [(320, 64), (70, 129), (8, 1000)])
def test_ranks_and_widths(N, K, R, x, w):
    print(N, K, R, x, w, flush=True)
    Call(131, N, K, R, *RAGGED, 3, x, w, seed=R).check()


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("M,starts,of", [
    (1, [0, 1], [0]),                                         # one token
    (64, list(range(65)), [i % 5 for i in range(64)]),        # a token and an adapter per request
    (300, [0, 300], [4]),                                     # one request
    (300, [7, 100, 100, 290], [1, 2, 3]),                     # rows of no request at both ends, an empty request
    (200, [0, 50, 100, 150, 200], [-1, 5, 1000, 3]),          # adapters that are none
    (90, [0, 0, 90, 90], [0, 0, 0]),
    (50, [], []),                                             # no request
])
def test_requests(M, starts, of, x, w):
    print(M, len(of), x, w, flush=True)
    Call(M, 96, 160, 16, starts or [0], of, 5, x, w, seed=M).check()


@pytest.mark.parametrize("x,w", PAIRS)
def test_more_requests_than_are_looked_over_at_once(x, w):
    rng = np.random.default_rng(3)
    lengths = rng.integers(0, 4, 1300)
    starts = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    of = rng.integers(-1, 7, 1300).tolist()
    Call(starts[-1] + 5, 48, 64, 8, starts, of, 7, x, w).check()


@pytest.mark.parametrize("x,w", PAIRS)
def test_rows_cut_over_workgroups(x, w):
    """Gradients joined from parts of the rows, tiles of 16 and of 32 rows."""
    Call(5000, 160, 320, 16, [0, 1234, 5000], [1, 0], 2, x, w).check()
    Call(40, 64, 2560, 16, [0, 20, 40], [0, 1], 2, x, w).check()
    Call(16500, 40, 64, 16, [0, 7000, 16431], [0, 1], 2, x, w).check()


def test_base_none_and_in_place_and_t_not_kept():
    for K in (96, 2560):
        c = Call(131, 320, K, 16, *RAGGED, 3)
        y, t = c.forward()
        inplace = c.base.clone()
        assert torch.equal(c.forward(base=inplace, y=inplace)[0], y)
        assert torch.equal(c.forward(keep_t=False)[0], y)
        zeros = torch.zeros_like(c.base)
        assert torch.equal(c.forward(base=None)[0], c.forward(base=zeros)[0])
        gx, ga, gb = c.backward(t)
        again = c.backward(t, gx=None)
        assert again[0] is None and torch.equal(again[1], ga) and torch.equal(again[2], gb)
        inplace = c.gx_base.clone()
        assert torch.equal(c.backward(t, base=inplace, gx=inplace)[0], gx)
        assert torch.equal(c.backward(t, base=None)[0], c.backward(t, base=torch.zeros_like(c.x))[0])
        assert torch.equal(y[66:130], c.base[66:130]) and torch.all(t[66:130] == 0) and torch.equal(gx[66:130], c.gx_base[66:130])


def test_strides_and_alignment():
    for x, w in PAIRS:
        c = Call(131, 320, 96, 16, *RAGGED, 3, x, w)
        y, t = c.forward()
        gx, ga, gb = c.backward(t)
        for pad, shift in ((8, 0), (3, 0), (5, 1)):
            def place(z):
                flat = nan(shift + z.shape[0] * (z.shape[1] + pad), t=z.dtype)
                v = flat[shift:].view(z.shape[0], -1)[:, :z.shape[1]]
                v.copy_(z)
                return flat, v
            wide = {n: place(getattr(c, n)) for n in ("x", "base", "gy", "gx_base")}
            d = Call(131, 320, 96, 16, *RAGGED, 3, x, w)
            for n, (_, v) in wide.items():
                setattr(d, n, v)
            out, view = place(torch.zeros_like(c.base))
            got, _ = d.forward(y=view)
            assert torch.equal(got, y)
            assert torch.isnan(out[shift:].view(131, -1)[:, 320:]).all()
            out, view = place(torch.zeros_like(c.x))
            got = d.backward(t, gx=view)
            assert torch.equal(got[0], gx) and torch.equal(got[1], ga) and torch.equal(got[2], gb)
            assert torch.isnan(out[shift:].view(131, -1)[:, 96:]).all()


def test_bits_repeat_and_do_not_depend_on_other_requests():
    c = Call(131, 320, 96, 16, *RAGGED, 3)
    first = [*c.forward(), *c.backward(c.forward()[1])]
    again = [*c.forward(), *c.backward(c.forward()[1])]
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    d = Call(131, 320, 96, 16, *RAGGED, 3)
    d.x[34:66] = float("nan")                                  # the request of adapter 1, and nobody else's
    y, t = d.forward()
    keep = [i for i in range(131) if not 34 <= i < 66]
    assert torch.equal(y[keep], first[0][keep]) and torch.isnan(y[34:66]).all()
    _, ga, gb = d.backward(t)
    assert torch.equal(ga[[0, 2]], first[3][[0, 2]]) and torch.equal(gb[[0, 2]], first[4][[0, 2]])


def test_another_stream_and_a_graph():
    c = Call(131, 320, 96, 16, *RAGGED, 3)
    y, t = c.forward()
    want = [y, t, *c.backward(t)]
    bufs = [torch.full_like(z, float("nan")) for z in want]
    ws = room(max(B.fpq_adapter_workspace_size(*c.sizes), B.fpq_adapter_backward_workspace_size(*c.sizes)))

    def call():
        B.fpq_adapter_apply(*c.shared, c.base, bufs[0], bufs[1], ws)
        B.fpq_adapter_backward(*c.shared, bufs[1], c.gy, c.gx_base, *bufs[2:], ws)

    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(bufs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for z in bufs:
            z.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bufs, want))


@pytest.mark.parametrize("x,w", PAIRS)
def test_more_requests_than_a_list_holds(x, w):
    """Requests of one row, of none and of many, in several lists; an adapter's rows in all of them, another's in the last only."""
    starts = [0]
    for i in range(1300):
        starts.append(starts[-1] + (0 if i % 7 == 3 else 70 if i % 400 == 5 else 1))
    of = [2 if i >= 1200 and i % 5 == 0 else i % 2 if i % 3 else -1 for i in range(1300)]
    Call(starts[-1] + 20, 72, 40, 8, starts, of, 4, x, w).check()
