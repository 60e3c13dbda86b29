"""append_quantized over all exponents and signs of a type: every 16-bit pattern, and some million f32 ones, as blocks of alike and of different magnitudes, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk
from oracle import quant as oracle

pytestmark = pytest.mark.gpu


def same_rows(x, bits):
    """x (tokens, 1, dim): what append leaves in a pool against the ladder's codes and exponents."""
    tokens, heads, dim = x.shape
    ps = 64
    pages = -(-tokens // ps)
    t = atk.PageTables.empty(pages, ps, 1, pages)
    pool = torch.zeros((pages, ps, atk.quantized_token_bytes(heads, dim, bits)), dtype=torch.uint8, device="cuda")
    atk.append_quantized(t, [pool], torch.zeros((1,), dtype=torch.int32, device="cuda"), [x.cuda()[None]], bits=bits)
    assert t.status.item() == 0
    got = pool[t.page_table[0].long()].reshape(pages * ps, -1)[:tokens].cpu().numpy()
    want = oracle.encode(x.double().numpy(), bits)
    wrong = np.nonzero((got != want).any(1))[0]
    assert wrong.size == 0, (wrong.size, x[wrong[0]].tolist(), got[wrong[0]].tolist(), want[wrong[0]].tolist())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_every_pattern(bits, dtype):
    every = torch.arange(-(1 << 15), 1 << 15, dtype=torch.int32).to(torch.int16).view(dtype)
    every = every[torch.isfinite(every)]
    every = every[:every.numel() // 256 * 256]
    order = torch.argsort(every.float().abs(), stable=True)
    for x in (every[order], every[torch.randperm(every.numel(), generator=torch.Generator().manual_seed(0))]):     # alike, different
        same_rows(x.reshape(-1, 1, 256), bits)
    # each as a block of its own, beside smaller ones
    x = every[order][:, None].float() * torch.exp2(-torch.arange(32.0) * 0.5)[None, :]
    same_rows(x.to(dtype).reshape(-1, 1, 256), bits)


@pytest.mark.parametrize("bits", [4, 8])
def test_f32(bits):
    g = torch.Generator().manual_seed(1)
    n = 1 << 22
    some = torch.randint(-(1 << 31), 1 << 31, (n,), generator=g, dtype=torch.int64).to(torch.int32).view(torch.float32)
    some = torch.where(torch.isfinite(some), some, 1.0)
    same_rows(some[torch.argsort(some.abs())].reshape(-1, 1, 256), bits)       # blocks of alike ones, all exponents, subnormal numbers too
    same_rows(some[:1 << 20].reshape(-1, 1, 256), bits)
    # blocks over the format's range, of every exponent; middles between codes and their neighbours
    low = torch.randint(0, 13 if bits == 4 else 20, (n // 32, 32), generator=g)
    e = torch.arange(n // 32) % 254 + 1
    mantissa = torch.randint(0, 1 << 23, (n // 32, 32), generator=g)
    coarse = torch.randint(0, 16, (n // 32, 32), generator=g) << 19
    coarse = (coarse + torch.randint(-1, 2, (n // 32, 32), generator=g)).clamp(0, (1 << 23) - 1)
    mantissa = torch.where(torch.rand((n // 32, 32), generator=g) < 0.5, coarse, mantissa)
    exponent = (e[:, None] - low).clamp(0, 254)
    sign = torch.randint(0, 2, (n // 32, 32), generator=g)
    x = ((sign << 31) | (exponent << 23) | mantissa).to(torch.int64)
    x = torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32).view(torch.float32)
    same_rows(x.reshape(-1, 1, 256), bits)
