"""shared_prefix_attention at the ends of the scales that it takes: the lse is the log of the number of keys where all weights are alike."""
import math

import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
@pytest.mark.parametrize("B,H,Hk,keys,prefix,room", [(2, 4, 2, 160, 64, 0), (3, 4, 2, 2048, 1024, 0), (70, 8, 2, 1536, 1024, 0), (600, 8, 8, 1024, 1024, 0)], ids=str)
@pytest.mark.parametrize("scale", [1.1754943508222875e-38, 1e-30])
def test_smallest_scales(dtype, B, H, Hk, keys, prefix, room, scale):
    g = torch.Generator(device="cuda").manual_seed(keys)
    table = torch.arange(keys // 16, dtype=torch.int32, device="cuda").repeat(B, 1)
    k, v = (torch.randn((keys // 16, 16, Hk, 64), generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn((B, 1, H, 64), generator=g, device="cuda").to(dtype)
    lens = torch.full((B,), keys, dtype=torch.int32, device="cuda")
    out, lse = atk.shared_prefix_attention(q, k, v, table, lens, prefix, scale=scale, return_lse=True)
    want = v.double().reshape(keys, Hk, 64).mean(0).repeat_interleave(H // Hk, 0)
    # all weights are 1: sums over the keys in f32, and the result's rounding
    h = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}[dtype]
    assert (out.double() - want).abs().max().item() <= h * want.abs().max().item() + 2.0 ** -24 * (8 + 2 * keys) * v.double().abs().mean().item() * 4 + (2.0 ** -24 if dtype == torch.float16 else 0.0)
    assert (lse.double() - math.log(keys)).abs().max().item() <= 2.0 ** -24 * (keys + 4 * (1 + math.log(keys)))
    with pytest.raises(atk.ApproxTopkError):
        atk.shared_prefix_attention(q, k, v, table, lens, prefix, scale=1e-46, return_lse=True)
