"""Results written into a tensor of the caller's: autograd hears of it, as of torch's own operations in place."""
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu


def test_gradient_in_the_logits_place():
    x = torch.randn((1, 2, 300), device="cuda", requires_grad=True)
    y = torch.tanh(x)                      # (whose backward needs y as it was)
    tokens = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    one = torch.ones((1, 2), device="cuda")
    _, h, lse, _, _ = atk.token_logprobs(y, tokens)
    want = torch.autograd.grad(y, x, atk.token_logprobs_grad(y, tokens, lse, h, one, one), retain_graph=True)[0]
    assert torch.isfinite(want).all()
    flat = y.detach()
    g = atk.token_logprobs_grad(flat, tokens, lse, h, one, one, out=flat)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(g)


def test_gradient_in_a_tensor_that_backward_needs():
    x = torch.randn((1, 1, 50), device="cuda", requires_grad=True)
    buffer = torch.empty((1, 1, 50), device="cuda")
    z = x * buffer.fill_(2.0)              # (whose backward needs the buffer)
    tokens, one = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.ones((1, 1), device="cuda")
    lse = atk.token_logprobs(z, tokens)[2]
    atk.token_logprobs_grad(z, tokens, lse, None, one, out=buffer)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.sum().backward()


@pytest.mark.parametrize("pages", [3, 0])
def test_attention(pages):
    size = atk.quantized_token_bytes(1, 64)
    pool = torch.zeros((pages, 16, size), dtype=torch.uint8, device="cuda")
    q, out = torch.randn((1, 1, 2, 64), device="cuda"), torch.ones((1, 1, 2, 64), device="cuda")
    table, lens = torch.zeros((1, 3), dtype=torch.int32, device="cuda"), torch.full((1,), 20, dtype=torch.int32, device="cuda")
    x = torch.ones((1, 1, 2, 64), device="cuda", requires_grad=True)
    z = x * out
    assert atk.quantized_attention(q, pool, pool, table, lens, 1, out=out) is out
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.sum().backward()
    with torch.inference_mode():
        atk.quantized_attention(q, pool, pool, table, lens, 1, out=torch.empty_like(q))
