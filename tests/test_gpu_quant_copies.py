"""Quantised pages handed from one cache to another, under other numbers: the same bytes, and the same attention."""
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("heads,dim", [(2, 64), (3, 96), (1, 256)])
def test_pages_go_to_another_cache(bits, heads, dim):
    g = torch.Generator().manual_seed(heads)
    size = atk.quantized_token_bytes(heads, dim, bits)
    t = atk.PageTables.empty(12, 16, 2, 6)
    pools = [torch.zeros((12, 16, size), dtype=torch.uint8, device="cuda") for _ in range(2)]
    atk.append_quantized(t, pools, ints(0, 1), [torch.randn((2, 75, heads, dim), generator=g).bfloat16().cuda() for _ in range(2)], bits=bits)
    q = torch.randn((2, 2, 2 * heads, dim), generator=g).bfloat16().cuda()
    want = atk.quantized_attention(q, *pools, t.page_table, t.lens, heads, bits=bits, status=t.status)
    far = [torch.full((40, 16, size), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    src = t.page_table[t.page_table >= 0]
    dst = (torch.randperm(28, generator=g)[:src.numel()] + 12).int().cuda()
    status = ints(0)
    atk.copy_pages(pools, src, far, dst, status=status)
    table = t.page_table.clone()
    table[table >= 0] = dst
    assert torch.equal(atk.quantized_attention(q, *far, table, t.lens, heads, bits=bits, status=status), want)
    assert status.item() == 0 and t.status.item() == 0
    rest = torch.ones(40, dtype=torch.bool)
    rest[dst.cpu().long()] = False
    assert all((pool[rest.cuda()] == 255).all() for pool in far)
