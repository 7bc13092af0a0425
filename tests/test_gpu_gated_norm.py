"""bf16 gradients of gated projections in norm: no further from the rounded result in 64 bits than operands of 16 bits make them."""
import pytest

from oracle import adapt, blocks
from test_gpu_blocks import E4M3, host, quantize
from test_gpu_gated import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("keep", ["type", "blocks"])
@pytest.mark.parametrize("M,N,K", [(300, 160, 320), (257, 96, 160), (64, 200, 128), (500, 77, 65), (2100, 160, 1400), (17, 1000, 264), (3, 333, 72)])
def test_no_further_than_the_roundings(M, N, K, keep, act):
    """grad_x and grad_w together, each alone, and grad_w from blocks of x."""
    print(M, N, K, keep, act, flush=True)
    c = Call(M, N, K, "bf16", act)
    _, pre, scales = c.forward(keep)
    xq, xs = quantize(c.x, E4M3)
    kept = blocks.block_values(xq.cpu().numpy(), xs.cpu().numpy(), 8, K)
    a, g = c.kept_values(pre, scales)
    w, gh = host(c.w), host(c.gh)
    for name, x, args, which in (("both", host(c.x), (), (True, True)), ("grad_x", host(c.x), (), (True, False)), ("grad_w", host(c.x), (), (False, True)),
                                 ("blocks", kept, (xq, xs), (True, True))):
        got = c.backward(pre, scales, *args, gx=which[0], gw=which[1])[:2]
        want, spread = blocks.gated_backward(x, w, a, g, act, gh, True), blocks.gated_spread(x, w, a, g, act, gh)
        far = [adapt.off_in_norm(host(v), t[0], s) for v, t, s in zip(got, want, spread) if v is not None]
        print(name, ["%.3f" % f for f in far], flush=True)
        assert all(f <= 1 for f in far), (name, far)
