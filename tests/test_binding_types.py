"""Index and statistics tensors of another type, with elements of the same size, are refused by the binding: read as what they are
not they would be lengths past the buffer, adapters that do not exist, rows of no request.  No GPU needed."""
import pytest
import torch

from paper_2408_06995_amd import binding as B

I, F = torch.int32, torch.float32


def attention(**kw):
    q, k = torch.zeros(2, 8, 4, 16), torch.zeros(2, 9, 2, 16)
    a = dict(lse=torch.zeros(2, 4, 8), kv_lens=torch.zeros(2, dtype=I))
    a.update(kw)
    B.fpq_attention(q, k, k, q, a["lse"], 1.0, 0, a["kv_lens"])


def attention_backward(**kw):
    q, k = torch.zeros(2, 8, 4, 16), torch.zeros(2, 9, 2, 16)
    a = dict(lse=torch.zeros(2, 4, 8), kv_lens=torch.zeros(2, dtype=I))
    a.update(kw)
    B.fpq_attention_backward(q, k, k, q, a["lse"], q, q, k, k, 1.0, 0, a["kv_lens"])


def adapter(backward, **kw):
    x, y = torch.zeros(10, 64), torch.zeros(10, 32)
    a = dict(scaling=torch.ones(3), row_start=torch.zeros(3, dtype=I), adapter=torch.zeros(2, dtype=I), t=torch.zeros(10, 8), grad_a=torch.zeros(3, 8, 64),
             grad_b=torch.zeros(3, 32, 8))
    a.update(kw)
    shared = (x, torch.zeros(3, 8, 64), torch.zeros(3, 32, 8), a["scaling"], a["row_start"], a["adapter"])
    if backward:
        B.fpq_adapter_backward(*shared, a["t"], y, None, None, a["grad_a"], a["grad_b"])
    else:
        B.fpq_adapter_apply(*shared, None, y, a["t"])


def other(t):
    return t.view(F if t.dtype == I else I)


@pytest.mark.parametrize("name,value", [("lse", torch.zeros(2, 4, 8)), ("kv_lens", torch.zeros(2, dtype=I))])
@pytest.mark.parametrize("call", [attention, attention_backward])
def test_attention(call, name, value):
    with pytest.raises(TypeError, match=name):
        call(**{name: other(value)})


@pytest.mark.parametrize("backward,name,value", [
    (b, n, v) for b in (False, True) for n, v in (("scaling", torch.ones(3)), ("row_start", torch.zeros(3, dtype=I)), ("adapter", torch.zeros(2, dtype=I)),
                                                  ("t", torch.zeros(10, 8)), ("grad_a", torch.zeros(3, 8, 64)), ("grad_b", torch.zeros(3, 32, 8)))
    if b or not n.startswith("grad")])
def test_adapter(backward, name, value):
    with pytest.raises(TypeError, match=name):
        adapter(backward, **{name: other(value)})


def test_adamw_scale_of_the_gradient():
    with pytest.raises(TypeError, match="grad_scale"):
        B.fpq_adamw_step(torch.zeros(96, dtype=torch.uint8), 0, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1, torch.zeros(1, dtype=I))
