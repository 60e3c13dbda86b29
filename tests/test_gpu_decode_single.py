"""shared_prefix_attention on tensors with a dimension of one element, whose stride says nothing."""
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_one_sequence_out_of_rows_of_odd_width(dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((8, 16, 2, 64), generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn((1, 3, 4, 64), generator=g, device="cuda").to(dtype)
    table, lens = torch.arange(8, dtype=torch.int32, device="cuda").reshape(1, 8), torch.tensor([100], dtype=torch.int32, device="cuda")
    wide = torch.zeros((2, 3 * 4 * 64 + 3), dtype=dtype, device="cuda")
    odd = torch.as_strided(wide, (2, 3, 4, 64), (3 * 4 * 64 + 3, 256, 64, 1))[:1]
    odd.copy_(q)
    assert odd.stride(0) % 2
    pages = torch.as_strided(k, (1, 16, 2, 64), (7, 128, 64, 1))
    one = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    for out in (None, torch.as_strided(torch.zeros_like(wide), (2, 3, 4, 64), (3 * 4 * 64 + 3, 256, 64, 1))[:1]):
        assert torch.equal(atk.shared_prefix_attention(odd, k, v, table, lens, 40, out=out), atk.shared_prefix_attention(q, k, v, table, lens, 40))
        lens[0] = 16
        assert torch.equal(atk.shared_prefix_attention(odd, pages, pages, one, lens, 0, out=out), atk.shared_prefix_attention(q, k, k, table, lens, 0))
        lens[0] = 100
