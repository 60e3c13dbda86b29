"""shared_prefix_attention of many rows on shared keys: what only the device sees and is out of range is reported, and means the same, whichever kernel meets it."""
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def made(B, Hk, G, D, prefix, ps, dtype, T=1, more=0, seed=0):
    """Shared keys alone fill the rows of the table, or `more` pages stand behind them."""
    g = torch.Generator(device="cuda").manual_seed(seed + prefix)
    shared = prefix // ps
    P = shared + B * more
    ids = torch.randperm(P, generator=g, device="cuda").int()
    table = torch.cat([ids[:shared].repeat(B, 1), ids[shared:].reshape(B, more)], 1).contiguous()
    k, v = (torch.randn((P, ps, Hk, D), generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn((B, T, Hk * G, D), generator=g, device="cuda").to(dtype)
    return q, k, v, table


# few rows (one kernel on all keys), and many: one range, several, eight wavefronts
SIZES = [(8, 2, 2, 64, 1024, 16), (600, 8, 1, 128, 1024, 16), (130, 4, 1, 128, 1024, 16), (300, 4, 2, 64, 4096, 32)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_lengths_past_a_row_that_shared_keys_fill(dtype, size):
    B, prefix = size[0], size[4]
    q, k, v, table = made(*size, dtype)
    lens = torch.full((B,), prefix, dtype=torch.int32, device="cuda")
    status = ints([0])
    want = atk.shared_prefix_attention(q, k, v, table, lens, prefix, status=status)
    assert status.item() == 0
    for at in (0, B // 2, B - 1):
        for length in (prefix + 1, (1 << 31) - 1):
            bad = lens.clone()
            bad[at] = length
            got = atk.shared_prefix_attention(q, k, v, table, bad, prefix, status=status)
            assert status.item() == atk.ATK_STATUS_BAD_LEN and torch.equal(got, want)   # as long as the row can be
            status.zero_()
    bad = lens.clone()
    bad[B - 2] = -1
    got = atk.shared_prefix_attention(q, k, v, table, bad, prefix, status=status)
    assert status.item() == atk.ATK_STATUS_BAD_LEN and (got[B - 2] == 0).all()
    status.zero_()
    seqs = torch.arange(B, dtype=torch.int32, device="cuda")
    seqs[B - 1] = B
    got = atk.shared_prefix_attention(q, k, v, table, lens, prefix, seqs=seqs, status=status)
    assert status.item() == atk.ATK_STATUS_BAD_SEQ and (got[B - 1] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("more", [0, 1, 40])
def test_keys_of_pages_that_are_none(dtype, size, more):
    # as if they were not there: the same keys without them, in rows that are shorter by these pages
    B, Hk, G, D, prefix, ps = size
    q, k, v, table = made(*size, dtype, more=more, seed=3)
    lens = prefix + torch.randint(0, more * ps + 1, (B,), generator=torch.Generator().manual_seed(1)).int().cuda()
    none = sorted({0, 5, prefix // ps // 2, prefix // ps - 1})
    bad = table.clone()
    bad[0, none] = ints([1 << 30, -1, -(1 << 31), k.shape[0]])[:len(none)]    # only the first row's are read
    status = ints([0])
    out, lse = atk.shared_prefix_attention(q, k, v, bad, lens, prefix, return_lse=True, status=status)
    assert status.item() == atk.ATK_STATUS_BAD_PAGE
    held = [j for j in range(table.shape[1]) if j not in none]
    gone = len(none) * ps
    want, wlse = atk.shared_prefix_attention(q, k, v, table[:, held].contiguous(), lens - gone, prefix - gone, return_lse=True)
    # Either is off by its roundings, counted as in test_gpu_decode_attention.py: h half a step of the type, e = 2^-24; the weights add up to 1, and no value is above `big`.
    h = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}[dtype]
    e, n, big, scale = 2.0 ** -24, prefix + more * ps, v.double().abs().max().item(), D ** -0.5
    size = max((q[:, :, i * G:(i + 1) * G].reshape(-1, D).float().abs() @ k[:, :, i].reshape(-1, D).float().abs().t().contiguous()).max().item() for i in range(Hk)) * scale
    weight = 2 * (D + 4) * e * size + (4 + n) * e
    tol = big * (2 * h + 2 * weight) + (2 * n * big * 2.0 ** -31 + 2.0 ** -24 if dtype == torch.float16 else 0.0)
    assert (out.double() - want.double()).abs().max().item() <= 2 * tol
    assert (lse.double() - wlse.double()).abs().max().item() <= 2 * (weight + 4 * e * (1 + wlse.abs().max().item()))
