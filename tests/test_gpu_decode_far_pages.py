"""shared_prefix_attention of many rows on shared keys in pages 2^32 bytes and more apart: offsets of 16 bytes in 32 bits up to the limit of those, another kernel past it.

The tolerance is that of test_gpu_decode_attention.py: h half a step of the type, e = 2^-24."""
import ctypes

import pytest
import torch

import paper_2412_04358_amd as atk
from paper_2412_04358_amd import decode

pytestmark = pytest.mark.gpu
LIMIT = 1 << 31   # elements from page to page of a cache of eight: 2^34 of all of them
PAGES = 8


def parts(B, H, Hk, D, ps, prefix, stride):
    i3 = ctypes.c_int64 * 3
    q, k = i3(H * D, H * D, D), i3(stride, Hk * D, D)
    a = decode._AttentionArgs(batch=B, tokens=1, heads=H, kv_heads=Hk, dim=D, page_size=ps, n_pages=PAGES, rows=B, row_pages=PAGES, table_stride=PAGES, prefix_len=prefix, q_stride=q,
                              out_stride=q, k_stride=k, v_stride=k, scale=1.0, dtype=atk.ATK_BF16)
    return decode._library().atk_attention_workspace_bytes(a) // (B * H * (4 * D + 8))


@pytest.fixture(scope="module")
def memory():
    buffer = torch.empty((PAGES * (LIMIT + 8) + (1 << 21),), dtype=torch.bfloat16, device="cuda")
    yield buffer
    del buffer
    torch.cuda.empty_cache()


@pytest.mark.parametrize("more", [0, 8], ids=["limit", "past"])
@pytest.mark.parametrize("B,H,Hk,D,ps", [(300, 8, 2, 128, 256), (600, 4, 4, 128, 256), (70, 8, 2, 64, 256), (40, 8, 2, 256, 1024)], ids=str)
def test_far_pages(memory, B, H, Hk, D, ps, more):
    g = torch.Generator(device="cuda").manual_seed(D + B)
    stride = LIMIT + more
    near = [torch.randn((PAGES, ps, Hk, D), generator=g, device="cuda").bfloat16() for _ in range(2)]
    far = [torch.as_strided(memory, (PAGES, ps, Hk, D), (stride, Hk * D, D, 1), offset) for offset in (0, 1 << 20)]
    assert ps * Hk * D <= 1 << 20
    for a, b in zip(far, near):
        a.copy_(b)
    prefix, n = 7 * ps, 8 * ps
    table = torch.randperm(PAGES, generator=g, device="cuda").int().repeat(B, 1)
    lens = torch.randint(prefix, n + 1, (B,), generator=g, device="cuda").int()
    q = torch.randn((B, 1, H, D), generator=g, device="cuda").bfloat16()
    out, lse = atk.shared_prefix_attention(q, *far, table, lens, prefix, return_lse=True)
    if not more:
        want, wlse = atk.shared_prefix_attention(q, *near, table, lens, prefix, return_lse=True)
        assert parts(B, H, Hk, D, ps, prefix, stride) == parts(B, H, Hk, D, ps, prefix, ps * Hk * D)   # the same plan, so the same bits
        assert torch.equal(out, want) and torch.equal(lse, wlse)
    elif B == 300:
        assert parts(B, H, Hk, D, ps, prefix, stride) != parts(B, H, Hk, D, ps, prefix, ps * Hk * D)
    h, e, G = 2.0 ** -8, 2.0 ** -24, H // Hk
    sees = (torch.arange(n, device="cuda")[None, :] < lens[:, None]).repeat_interleave(G, 0)
    for head in range(Hk):
        k, v = (x[table[0].long(), :, head].reshape(n, D).double() for x in near)
        qq = q[:, 0, head * G:(head + 1) * G].reshape(-1, D).double()
        s = (qq @ k.t().contiguous() * D ** -0.5).masked_fill(~sees, float("-inf"))
        wlse = torch.logsumexp(s, 1)
        w = torch.exp(s - wlse[:, None])
        want, mass = w @ v, w @ v.abs()
        weight = 2 * (D + 4) * e * D ** -0.5 * (qq.abs() @ k.abs().t().contiguous()).amax(1) + (4 + n) * e
        got, got_lse = out[:, 0, head * G:(head + 1) * G].reshape(-1, D).double(), lse[:, 0, head * G:(head + 1) * G].reshape(-1).double()
        assert ((got - want).abs() <= mass * (h + 2 * weight)[:, None] + h * want.abs()).all()
        assert ((got_lse - wlse).abs() <= weight + 4 * e * (1 + wlse.abs())).all()
