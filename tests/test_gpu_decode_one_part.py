"""shared_prefix_attention where the shared keys fill the rows of the table and are one range: nothing is joined, the kernel of many rows writes the results itself.  Against products in 64 bits on the GPU.

Tolerances as in test_gpu_decode_attention.py: h half a step of the type, e = 2^-24; weights and results are rounded to the type, scores are sums of dim products in f32, 2^x is good
to 4 e, sums over n keys add n e; f16 weights have steps of 2^-31 of the largest."""
import ctypes

import pytest
import torch

import paper_2412_04358_amd as atk
from paper_2412_04358_amd import decode

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
E = 2.0 ** -24


def planned_bytes(q, k, table, prefix):
    """Bytes of the call's workspace: 4 * dim + 8 for each part of a row."""
    B, T, H, D = q.shape
    P, ps, Hk, _ = k.shape
    i3 = ctypes.c_int64 * 3
    a = decode._AttentionArgs(batch=B, tokens=T, heads=H, kv_heads=Hk, dim=D, page_size=ps, n_pages=P, rows=table.shape[0], row_pages=table.shape[1], table_stride=table.stride(0),
                              prefix_len=prefix, q_stride=i3(*q.stride()[:3]), out_stride=i3(*q.stride()[:3]), k_stride=i3(*k.stride()[:3]), v_stride=i3(*k.stride()[:3]), scale=1.0,
                              dtype=atk.ATK_F16 if q.dtype == torch.float16 else atk.ATK_BF16)
    return decode._library().atk_attention_workspace_bytes(a)


@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("B,T,H,Hk,D,ps", [
    (600, 1, 32, 32, 128, 16), (1024, 1, 32, 8, 128, 16), (1024, 1, 32, 8, 96, 64),   # four wavefronts
    (257, 1, 128, 128, 64, 16), (512, 1, 64, 64, 64, 32), (300, 1, 96, 96, 72, 8),    # eight
    (128, 8, 32, 8, 128, 16), (600, 1, 32, 32, 256, 16),
], ids=str)
@pytest.mark.parametrize("short", [False, True], ids=["all", "short"])
def test_one_range_and_no_room_for_own_keys(dtype, B, T, H, Hk, D, ps, short):
    prefix, G = 1024, H // Hk
    g = torch.Generator(device="cuda").manual_seed(B + D)
    P = prefix // ps
    ids = torch.randperm(P, generator=g, device="cuda")
    table = ids.int().repeat(B, 1)
    k, v = (torch.randn((P, ps, Hk, D), generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn((B, T, H, D), generator=g, device="cuda").to(dtype)
    lens = torch.full((B,), prefix, dtype=torch.int32, device="cuda")
    if short:  # sequences that end inside the shared keys, at the last but one, and an empty one: their row blocks go another way
        lens[3], lens[B // 2], lens[B - 1] = prefix // 2, prefix - 1, 0
    assert planned_bytes(q, k, table, prefix) == B * T * H * (4 * D + 8)
    out = torch.full_like(q, float("nan"))
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    _, lse = atk.shared_prefix_attention(q, k, v, table, lens, prefix, out=out, return_lse=True, status=status)
    assert status.item() == 0
    again = atk.shared_prefix_attention(q, k, v, table, lens, prefix)    # marshalled by the extension module
    assert torch.equal(again, out)
    h = HALF[dtype]
    limit = (lens.long()[:, None] - (T - 1) + torch.arange(T, device="cuda")[None, :])[:, :, None].expand(B, T, G).reshape(-1)
    sees = torch.arange(prefix, device="cuda")[None, :] < limit[:, None]
    live = limit > 0
    for head in range(Hk):
        kk, vv = (x[ids, :, head].reshape(prefix, D).double() for x in (k, v))
        qq = q[:, :, head * G:(head + 1) * G].reshape(-1, D).double()
        s = (qq @ kk.t().contiguous() * D ** -0.5).masked_fill(~sees, float("-inf"))
        wlse = torch.logsumexp(s, 1)
        w = torch.exp(s - wlse[:, None]).masked_fill(~sees, 0.0)
        want, mass = w @ vv, w @ vv.abs()
        size = (qq.abs() @ kk.abs().t().contiguous() * D ** -0.5).masked_fill(~sees, 0.0).amax(1)
        weight = 2 * (D + 4) * E * size + (4 + prefix) * E
        tol = mass * (h + 2 * weight)[:, None] + h * want.abs()
        if dtype == torch.float16:
            tol = tol + 2 * prefix * vv.abs().max() * 2.0 ** -31 + 2.0 ** -24
        got, got_lse = out[:, :, head * G:(head + 1) * G].reshape(-1, D).double(), lse[:, :, head * G:(head + 1) * G].reshape(-1).double()
        assert ((got - want).abs() <= tol).all()
        assert ((got_lse - wlse)[live].abs() <= (weight + 4 * E * (1 + wlse.abs()))[live]).all()
        assert (got[~live] == 0).all() and (got_lse[~live] == float("-inf")).all()
