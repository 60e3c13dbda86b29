"""shared_prefix_attention on keys with scores of -inf whose values are not finite: a row of nothing else is empty, beside other keys 0 times such a value is NaN - however the keys are
cut into ranges."""
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu


def made(B, H, Hk, D, keys, prefix, dtype, room):
    ps = 16
    g = torch.Generator(device="cuda").manual_seed(keys + B)
    shared, own = prefix // ps, (keys - prefix) // ps
    table = torch.full((B, keys // ps + room // ps), -1, dtype=torch.int32, device="cuda")
    ids = torch.randperm(shared + B * own, generator=g, device="cuda").int()
    table[:, :shared] = ids[:shared]
    table[:, shared:shared + own] = ids[shared:].reshape(B, own)
    k, v = (torch.randn((ids.numel(), ps, Hk, D), generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn((B, 1, H, D), generator=g, device="cuda").abs().to(dtype)    # (a score with a key of -inf is -inf)
    return q, k, v, table, torch.full((B,), keys, dtype=torch.int32, device="cuda")


# all in one launch; shared keys of few rows, with and without parts to join; many rows, mixed and apart; no own keys
@pytest.mark.parametrize("B,H,Hk,D,keys,prefix,room", [(2, 4, 2, 64, 160, 64, 0), (3, 4, 2, 128, 2048, 1024, 0), (3, 4, 2, 128, 1024, 1024, 0), (1, 1, 1, 64, 128, 0, 2048),
                                                       (70, 8, 2, 64, 1536, 1024, 0), (600, 8, 8, 128, 1024, 1024, 0), (600, 8, 8, 128, 1040, 1024, 16)], ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_values_behind_scores_of_nothing(B, H, Hk, D, keys, prefix, room, dtype, value):
    q, k, v, table, lens = made(B, H, Hk, D, keys, prefix, dtype, room)
    # all keys of the first head of keys; of the others one page, the last or the first
    for page in (0, keys // 16 - 1):
        kk, vv = k.clone(), v.clone()
        kk[:, :, 0], vv[:, :, 0] = float("-inf"), value
        at = table[0, page].long()
        kk[at], vv[at] = float("-inf"), value
        out, lse = atk.shared_prefix_attention(q, kk, vv, table, lens, prefix, return_lse=True)
        G = H // Hk
        assert (out[:, :, :G] == 0).all() and (lse[:, :, :G] == float("-inf")).all()
        if Hk > 1:
            with_it = slice(0, B) if page * 16 < prefix else slice(0, 1)
            assert torch.isnan(out[with_it, :, G:]).all() and torch.isfinite(lse[:, :, G:]).all()
            rest = out[B if page * 16 < prefix else 1:, :, G:]
            assert torch.isfinite(rest).all()
