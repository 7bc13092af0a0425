"""Attention asks for the workspace that a call uses, and stays within it."""
import pytest
import torch

from paper_2408_06995_amd import binding as B
from test_gpu_attention import nan_like, room, sizes, tensors

pytestmark = pytest.mark.gpu


def up(n):
    return -(-n // 256) * 256


def run(q, k, v, go, ws_forward, ws_backward):
    o, lse = nan_like(q), torch.full((q.shape[0], q.shape[2], q.shape[1]), float("nan"), device=q.device)
    grads = [nan_like(x) for x in (q, k, v)]
    B.fpq_attention(q, k, v, o, lse, 0.125, 0, None, ws_forward)
    B.fpq_attention_backward(q, k, v, o, lse, go, *grads, 0.125, 0, None, ws_backward)
    return [o, lse, *grads]


@pytest.mark.parametrize("shape,t,forward,backward", [
    # nothing is packed and nothing cut: the rows' statistics alone
    ((8, 512, 512, 16, 16, 64), "bf16", 0, 8 * 16 * 16 * 256),
    # two parts of the keys, and of the queries
    ((4, 512, 512, 16, 16, 64), "bf16", up(2 * 4 * 16 * 512 * 64 * 4) + up(2 * 4 * 16 * 512 * 4),
     4 * 16 * 16 * 256 + up(2 * 4 * 16 * 512 * 64 * 4) + up(4 * 4 * 16 * 512 * 64 * 4)),
    # planes of k and v, in the gradient of q and grad_o too; under the causal rule the same sizes are cut into parts
    ((2, 2048, 2048, 8, 8, 96), "fp32", 2 * up(2 * 8 * 2048 * 96 * 6), 2 * 8 * 64 * 256 + 4 * up(2 * 8 * 2048 * 96 * 6)),
])
def test_exactly_what_is_used(shape, t, forward, backward):
    q, k, v, go = tensors(*shape, t, 95)
    assert forward < B.fpq_attention_workspace_size(*sizes(q, k)) and backward < B.fpq_attention_backward_workspace_size(*sizes(q, k))
    want = run(q, k, v, go, room(B.fpq_attention_workspace_size(*sizes(q, k))), room(B.fpq_attention_backward_workspace_size(*sizes(q, k))))
    guard = [torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device=q.device) for n in (forward, backward)]
    got = run(q, k, v, go, guard[0][:forward] if forward else None, guard[1][:backward])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.all(g[n:] == 0x5a) for g, n in zip(guard, (forward, backward)))
    with pytest.raises(B.FpqError):
        run(q, k, v, go, guard[0][:forward] if forward else None, guard[1][:backward - 1])
    if forward:
        with pytest.raises(B.FpqError):
            run(q, k, v, go, guard[0][:forward - 1], guard[1])


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_unaligned_tensors_are_packed_into_it(t):
    """Rows off 16 bytes: what is stated is enough, and the results are those of aligned rows."""
    q, k, v, go = tensors(2, 300, 260, 4, 4, 64, t, 96)
    want = run(q, k, v, go, room(B.fpq_attention_workspace_size(*sizes(q, k))), room(B.fpq_attention_backward_workspace_size(*sizes(q, k))))

    def shifted(x):
        flat = torch.zeros(x.numel() + 1, dtype=x.dtype, device=x.device)
        y = flat[1:].view(x.shape)
        y.copy_(x)
        return y

    n = B.fpq_attention_workspace_size(*sizes(q, k)), B.fpq_attention_backward_workspace_size(*sizes(q, k))
    guard = [torch.full((max(s, 16) + 4096,), 0x5a, dtype=torch.uint8, device=q.device) for s in n]
    got = run(*(shifted(x) for x in (q, k, v, go)), guard[0][:max(n[0], 16)], guard[1][:n[1]])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.all(g[max(s, 16):] == 0x5a) for g, s in zip(guard, n))
