"""token_logprobs_grad on rows that lie far from 0, whose lse in f32 says little of the logits' distances from it: all of the type's lowest or largest value, or ordinary ones moved.

Against the formula in 64 bits on probabilities from the rows' largest logit.  With e = 2^-24, p is off by (3 |log p| + 5) e through its own exponential and by delta = (4 + 3 (mean + 4) + chain + 20) e, and as
much again for the logarithm, through the row's sum, of chains of vocab / 256 terms; the entropy that is given counts as exact."""
import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
E = 2.0 ** -24


def check(got, x, chosen, a, b, h):
    """got, x (rows, vocab) f64, the others (rows)."""
    V = x.shape[1]
    d = x - x.max(1, keepdims=True)
    logp = d - np.log(np.exp(d).sum(1, keepdims=True))
    p = np.exp(logp)
    logp = np.where(p > 0, logp, 0.0)
    there = (chosen >= 0) & (chosen < V)
    a = np.where(there, a, 0.0)[:, None]
    b, h = b[:, None], h[:, None]
    hit = np.arange(V)[None, :] == chosen[:, None]
    want = a * hit - p * (a + b * (logp + h))
    size = np.abs(a) * hit + p * (np.abs(a) + np.abs(b) * (np.abs(logp) + np.abs(h)))
    mean = (p * np.abs(logp)).sum(1, keepdims=True)
    delta = 24 + 3 * (mean + 4) + V / 256 + 8
    # (the gradient by log p itself, b p, has the same error in log p as p relatively)
    off = (size + p * np.abs(b)) * (3 * np.abs(logp) + 12 + 2 * delta + 2 * np.log(V)) * E
    return want, off


def rows_of(kind, B, T, V, dtype, g):
    info = torch.finfo(dtype)
    x = (3 * torch.randn((B, T, V), generator=g)).to(dtype)
    if kind in ("lowest", "largest"):
        x[0] = info.min if kind == "lowest" else info.max
        x[0, 0, V // 2:] = -float("inf") if V > 1 else x[0, 0, 0]
    else:
        shift = {"above": 1.0, "below": -1.0}[kind] * (2.0 ** 14 if dtype is torch.float32 else 2.0 ** 11)
        x[0] = (3 * torch.randn((T, V), generator=g, dtype=torch.float64) + shift).to(dtype)
    return x


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("kind", ["lowest", "largest", "above", "below"])
@pytest.mark.parametrize("B,T,V,pad", [(1, 1, 1, 0), (2, 2, 300, 1), (2, 1, 8192, 0), (2, 2, 8193, 7), (3, 1, 40000, 0), (1, 1, 128256, 64)], ids=str)
def test_far_rows(dtype, kind, B, T, V, pad):
    g = torch.Generator().manual_seed(V)
    wide = torch.zeros((B, T, V + pad), dtype=dtype, device="cuda")
    x = wide[..., :V]
    x.copy_(rows_of(kind, B, T, V, dtype, g))
    tokens = torch.randint(0, V, (B, T), generator=g).int().cuda()
    tokens[0, 0] = 0
    tokens[B - 1, T - 1] = min(V - 1, 3) if V < 400 else V    # (padding)
    a, b = torch.randn((B, T), generator=g).cuda(), torch.randn((B, T), generator=g).cuda()
    _, h, lse, _, _ = atk.token_logprobs(x, tokens)
    rows = x.double().cpu().numpy().reshape(B * T, V)
    chosen = tokens.cpu().numpy().reshape(-1)
    some = [t.double().cpu().numpy().reshape(-1) for t in (a, b, h)]
    zero = np.zeros(B * T)
    step = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134 if dtype == torch.bfloat16 else 2.0 ** -126   # (subnormal numbers; f32's p is 0 there)
    far = (lse.abs() >= 1024).cpu().numpy().reshape(-1)
    assert far[:T].all() and (kind not in ("lowest", "largest") or not far[T:].any())
    for ga, gb, ha, hb in ((a, b, some[0], some[1]), (a, None, some[0], zero), (None, b, zero, some[1])):
        got = atk.token_logprobs_grad(x, tokens, lse, h if gb is not None else None, ga, gb).double().cpu().numpy().reshape(B * T, V)
        want, off = check(got, rows, chosen, ha, hb, some[2])
        # (rows that are not far go by the lse that is given, whose rounding their p has)
        off = off + np.where(far, 0.0, np.abs(lse.double().cpu().numpy().reshape(-1)) * E)[:, None] * (np.abs(want) + np.exp(-np.abs(rows - rows.max(1, keepdims=True))) * 4)
        assert (np.abs(got - want) <= off + HALF[dtype] * np.abs(want) + step).all()
    # in the logits' place
    want = atk.token_logprobs_grad(x, tokens, lse, h, a, b)
    assert torch.equal(atk.token_logprobs_grad(x, tokens, lse, h, a, b, out=x), want) and torch.equal(x, want)
    if pad:
        assert (wide[..., V:] == 0).all()


def test_an_lse_of_more_logits():
    """The halves of a vocabulary with the whole one's lse: what is missing from a half is no rounding."""
    V = 20000
    g = torch.Generator().manual_seed(0)
    x = (3 * torch.randn((1, 1, V), generator=g) + 5000.0).cuda()
    tokens = torch.tensor([[77]], dtype=torch.int32, device="cuda")
    a, b = torch.ones((1, 1), device="cuda"), torch.full((1, 1), 0.5, device="cuda")
    _, h, lse, _, _ = atk.token_logprobs(x, tokens)
    for part, chosen in ((x[..., :V // 2], 77), (x[..., V // 2:], -1)):
        got = atk.token_logprobs_grad(part, torch.full((1, 1), chosen, dtype=torch.int32, device="cuda"), lse, h, a if chosen >= 0 else None, b).double()
        l = part.double() - lse.double()[..., None]
        p = torch.exp(l)
        want = -p * ((1.0 if chosen >= 0 else 0.0) + 0.5 * (l + h.double()[..., None]))
        if chosen >= 0:
            want[..., chosen] += 1.0
        assert (got - want).abs().max() < 2.0 ** -20


def test_infinite_lse():
    """What no logits have is taken as it is: no probability."""
    x = torch.zeros((1, 1, 9000), device="cuda")
    one, inf = torch.ones((1, 1), device="cuda"), torch.full((1, 1), float("inf"), device="cuda")
    got = atk.token_logprobs_grad(x, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), inf, None, one)
    assert got[0, 0, 0] == 1 and (got[0, 0, 1:] == 0).all()
