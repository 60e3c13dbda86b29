"""token_logprobs and token_logprobs_grad against their definitions in 64 bits: types, lengths, strides, ties, masks, rows without anything.

Tolerances, with e = 2^-24.  A term e^(x - r) is off by 3 e of x - r (a difference, a product with log2 e and that constant) and 4 e for the exponential itself, relatively; what it weighs is counted by the
mean of |log p| and the reference's distance (4 at most).  A sum of n terms in chains and trees adds at most (chain + 20) e, chains of n / 1024 * 8 terms or fewer than 2 n / 256.  So Z is off
by delta = (4 + 3 (mean + 4) + chain + 20) e, log Z by as much absolutely (and by 2 e of itself, as every sum and difference behind it by e of its size); the entropy's second part is the sum of d e^d / Z, by
(2 delta + 2 e) of the mean of |d|.  The gradient's p is off by (3 |log p| + 5) e, and the given lse counts as exact."""
import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk
from oracle import scores as oracle

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
E = 2.0 ** -24


def make(B, T, V, dtype, seed=0, pad=0, spread=3.0, banned=0.0):
    g = torch.Generator().manual_seed(seed)
    x = (spread * torch.randn((B, T, V + pad), generator=g)).to(dtype)
    if banned:
        x[torch.rand((B, T, V + pad), generator=g) < banned] = -float("inf")
    tokens = torch.randint(0, V, (B, T), generator=g).int()
    return x.cuda()[:, :, :V], tokens.cuda()


def check(x, tokens, top):
    B, T, V = x.shape
    got = [t.double().cpu().numpy() for t in atk.token_logprobs(x, tokens, top=top)]
    torch.cuda.synchronize()
    picked, entropy, lse, best, order, mean = oracle.logprobs(x.double().cpu().numpy().reshape(B * T, V), tokens.cpu().numpy().reshape(-1), top)
    assert np.array_equal(got[4].reshape(B * T, top), order)
    chain = 2 * V / 256 + 8
    delta = (24 + 3 * (mean + 4) + chain) * E
    off_lse = delta + 3 * E * (1 + np.abs(np.where(np.isfinite(lse), lse, 0)) + mean + 8)
    off_h = off_lse + (2 * delta + 4 * E) * (mean + 8)
    for name, a, b, tol in (("logprobs", got[0], picked, off_lse), ("entropy", got[1], entropy, off_h), ("lse", got[2], lse, off_lse), ("top", got[3].reshape(B * T, top), best, off_lse[:, None])):
        a = a.reshape(b.shape)
        assert np.array_equal(np.isnan(a), np.isnan(b)), name
        fine = np.isfinite(b)
        assert np.array_equal(a[~fine & ~np.isnan(b)], b[~fine & ~np.isnan(b)]), name
        size = np.where(fine, np.abs(np.where(fine, b, 0)), 0)
        off = np.abs(np.where(fine, a, 0) - np.where(fine, b, 0))
        assert (off <= tol + 2 * E * size).all(), (name, off.max())
    return got


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("B,T,V,top,pad,banned", [
    (1, 1, 1, 1, 0, 0.0), (2, 3, 2, 2, 1, 0.0), (1, 2, 7, 0, 0, 0.0), (3, 1, 127, 5, 2, 0.0), (1, 1, 128, 32, 0, 0.0), (2, 2, 129, 20, 7, 0.0), (1, 3, 513, 3, 0, 0.3),
    (2, 1, 1000, 32, 24, 0.95), (1, 1, 4097, 20, 3, 0.0), (4, 1, 32000, 5, 0, 0.0), (1, 2, 32769, 20, 0, 0.2), (3, 1, 50257, 20, 7, 0.0), (1, 1, 128256, 32, 64, 0.9),
    (300, 1, 2049, 4, 1, 0.0), (70, 4, 40000, 2, 0, 0.0),
], ids=str)
def test_shapes(dtype, B, T, V, top, pad, banned):
    x, tokens = make(B, T, V, dtype, seed=V, pad=pad, banned=banned)
    if B * T * V > 1 << 21:    # (the oracle takes its time: some of the rows, over all of which the kernels are planned)
        got = atk.token_logprobs(x, tokens, top=top)
        rows = [0, B // 2, B - 1]
        want = atk.token_logprobs(x.clone(), tokens, top=top)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        some = check(x[rows], tokens[rows], top)
        assert np.allclose(some[2], got[2][rows].cpu().numpy(), atol=1e-5) and np.array_equal(some[4], got[4][rows].cpu().numpy())
        assert np.allclose(some[0], got[0][rows].cpu().numpy(), atol=1e-5) and np.allclose(some[1], got[1][rows].cpu().numpy(), atol=1e-5)
        return
    check(x, tokens, top)


@pytest.mark.parametrize("V", [300, 5000, 40000, 140000])
@pytest.mark.parametrize("kind", ["equal", "few values", "rising", "falling", "far apart", "one", "lowest", "none", "zeros"])
def test_ties_orders_and_masks(V, kind):
    g = torch.Generator().manual_seed(V)
    for dtype in (torch.bfloat16, torch.float32):
        x = {"equal": torch.full((V,), 1.5), "few values": torch.randint(0, 3, (V,), generator=g).float(), "rising": torch.arange(V) / 1000.0, "falling": -torch.arange(V) / 1000.0,
             "far apart": 30 * torch.randn((V,), generator=g), "one": torch.where(torch.arange(V) == V // 3, 2.0, -float("inf")),
             "lowest": torch.where(torch.rand((V,), generator=g) < 0.9, torch.finfo(dtype).min, torch.randn((V,), generator=g)), "none": torch.full((V,), -float("inf")),
             "zeros": torch.where(torch.arange(V) % 2 == 0, -0.0, 0.0)}[kind].to(dtype).reshape(1, 1, V).cuda()
        check(x, torch.tensor([[V // 3]], dtype=torch.int32, device="cuda"), 32)


def test_numbers_that_are_none_and_tokens_that_are_none():
    x, tokens = make(1, 8, 3000, torch.float32, seed=4)
    x[0, 0, 100] = float("nan")
    x[0, 1, 2999] = float("inf")
    x[0, 2] = float("nan")
    x[0, 3, 5] = torch.finfo(torch.float32).max
    x[0, 4, :] = torch.finfo(torch.float32).min
    x[0, 5, 7] = -float("inf")
    tokens[0] = torch.tensor([5, 6, 7, 5, 9, 7, -1, 3000], dtype=torch.int32)
    check(x, tokens, 20)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_confident_rows_and_strides(dtype):
    g = torch.Generator().manual_seed(1)
    wide = torch.randn((5, 3, 2000), generator=g).to(dtype)
    wide[..., 11] = 25.0
    wide[1, :, 11] = 9.0
    wide = wide.cuda()
    tokens = torch.full((3, 5), 11, dtype=torch.int32, device="cuda")
    check(wide.transpose(0, 1), tokens, 3)
    check(wide[:1].expand(3, 3, 2000), tokens[:, :3].contiguous(), 3)
    check(wide[:, :, 3:1500], torch.full((5, 3), 8, dtype=torch.int32, device="cuda"), 3)


def test_long_vocabularies():
    """Groups of minis: 2^24 tokens, ties of which more come into question than there is room for."""
    V = 1 << 24
    x = torch.zeros((1, 1, V), dtype=torch.bfloat16, device="cuda")
    tokens = torch.tensor([[V - 1]], dtype=torch.int32, device="cuda")
    p, h, lse, tp, tt = atk.token_logprobs(x, tokens, top=32)
    assert tt[0, 0].tolist() == list(range(32)) and abs(lse.item() - np.log(V)) < 1e-5 and abs(h.item() - np.log(V)) < 1e-4 and abs(p.item() + np.log(V)) < 1e-5
    at = torch.randperm(V, generator=torch.Generator().manual_seed(0))[:40].sort().values
    x[0, 0, at.cuda()] = 2.0
    x[0, 0, V - 1] = 3.0
    tt = atk.token_logprobs(x, tokens, top=32)[4]
    assert tt[0, 0].tolist() == [V - 1] + [i for i in at.tolist() if i != V - 1][:31]
    x[0, 0] = (torch.arange(V, device="cuda") // 4096).bfloat16()       # a rising row: all that is near the end
    want = torch.sort(x[0, 0].float(), descending=True, stable=True).indices[:32]
    assert torch.equal(atk.token_logprobs(x, tokens, top=32)[4][0, 0], want.int())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("B,T,V,pad,banned", [(1, 1, 1, 0, 0.0), (2, 3, 7, 1, 0.0), (1, 2, 8, 0, 0.0), (3, 2, 1000, 7, 0.3), (2, 2, 8191, 0, 0.0), (1, 3, 8200, 64, 0.9), (1, 2, 32000, 0, 0.0)], ids=str)
def test_grad(dtype, B, T, V, pad, banned):
    x, tokens = make(B, T, V, dtype, seed=V + 1, pad=pad, banned=banned)
    tokens[0, 0] = -1 if V > 1 else 0
    if V > 7:
        x[0, T - 1] = -float("inf")
    p, h, lse, _, _ = atk.token_logprobs(x, tokens)
    g = torch.Generator().manual_seed(2)
    a, b = torch.randn((B, T), generator=g).cuda(), torch.randn((B, T), generator=g).cuda()
    rows = x.double().cpu().numpy().reshape(B * T, V)
    args = [t.double().cpu().numpy().reshape(-1) for t in (lse, h)]
    chosen = tokens.cpu().numpy().reshape(-1)
    some = [t.double().cpu().numpy().reshape(-1) for t in (a, b)]
    zero = np.zeros(B * T)
    with np.errstate(invalid="ignore"):
        logp = np.where(np.isfinite(rows) & np.isfinite(args[0])[:, None], np.abs(rows - args[0][:, None]), 0)
    for ga, gb, ha, hb in ((a, b, *some), (a, None, some[0], zero), (None, b, zero, some[1])):
        got = atk.token_logprobs_grad(x, tokens, lse, h if gb is not None else None, ga, gb)
        want, size = oracle.grad(rows, chosen, *args, ha, hb)
        off = np.abs(got.double().cpu().numpy().reshape(B * T, V) - want)
        step = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134 if dtype == torch.bfloat16 else 2.0 ** -126   # (subnormal numbers; f32's p is 0 there)
        assert (off <= size * (3 * logp + 12) * E + HALF[dtype] * np.abs(want) + step).all()
    # in the logits' place, and in rows of a wider tensor
    want = atk.token_logprobs_grad(x, tokens, lse, h, a, b)
    wide = torch.full((T, B, V + 5), 7.0, dtype=dtype, device="cuda")
    view = wide[:, :, 2:V + 2].transpose(0, 1)
    assert torch.equal(atk.token_logprobs_grad(x, tokens, lse, h, a, b, out=view), want) and (wide[:, :, :2] == 7).all() and (wide[:, :, V + 2:] == 7).all()
    assert torch.equal(atk.token_logprobs_grad(x, tokens, lse, h, a, b, out=x), want) and torch.equal(x, want)


def test_grad_against_differences():
    x, tokens = make(1, 2, 40, torch.float32, seed=9, spread=1.0)
    a, b = torch.tensor([[0.7, -1.3]], device="cuda"), torch.tensor([[0.4, 2.0]], device="cuda")
    _, h, lse, _, _ = atk.token_logprobs(x, tokens)
    got = atk.token_logprobs_grad(x, tokens, lse, h, a, b)
    step = 2.0 ** -6

    def value(y):
        p, e, *_ = atk.token_logprobs(y, tokens)
        return (a * p + b * e).double()

    for i in range(40):
        d = torch.zeros_like(x)
        d[..., i] = step
        # second-order differences are off by step^2 / 6 of a third derivative (below 10 here), the values by 2^-20 / step
        assert ((value(x + d) - value(x - d)) / (2 * step) - got[..., i].double()).abs().max() < step ** 2 / 6 * 10 + 2.0 ** -20 / step


def test_numbers_that_are_none_have_gradients_that_are_none():
    x, tokens = make(1, 3, 500, torch.float32, seed=4)
    x[0, 0, 100] = float("nan")
    x[0, 1, 5] = float("inf")
    p, h, lse, _, _ = atk.token_logprobs(x, tokens)
    one = torch.ones((1, 3), device="cuda")
    got = atk.token_logprobs_grad(x, tokens, lse, h, one, one)
    assert got[0, :2].isnan().all() and torch.isfinite(got[0, 2]).all()


def test_nothing_and_refusals():
    x, tokens = make(2, 3, 50, torch.float32)
    assert [tuple(t.shape) for t in atk.token_logprobs(x[:0], tokens[:0], top=2)] == [(0, 3)] * 3 + [(0, 3, 2)] * 2
    f = torch.zeros((2, 3), device="cuda")
    assert atk.token_logprobs_grad(x[:, :0], tokens[:, :0], f[:, :0], None, f[:, :0]).shape == (2, 0, 50)
    for args, kw, error in (((x, tokens.long()), {}, TypeError), ((x, tokens[:1]), {}, ValueError), ((x, tokens), dict(top=33), ValueError), ((x, tokens), dict(top=-1), ValueError), ((x[..., ::2], tokens), {}, ValueError),
                            ((x[..., :3], tokens), dict(top=4), ValueError), ((x[..., :0], tokens), {}, ValueError), ((x, tokens.cpu()), {}, ValueError)):
        with pytest.raises(error):
            atk.token_logprobs(*args, **kw)
    for args, kw, error in (((x, tokens, f.double(), f, f), {}, TypeError), ((x, tokens, f[:1], f, f), {}, ValueError), ((x, tokens, f, None, f, f), {}, ValueError), ((x, tokens, f, f, f), dict(out=x.half()), ValueError),
                            ((x, tokens, f, f, f), dict(out=x[:1].expand(2, 3, 50)), atk.ApproxTopkError)):
        with pytest.raises(error):
            atk.token_logprobs_grad(*args, **kw)


def test_captured_and_replayed():
    for B, V in ((3, 5000), (2, 60000)):
        x, tokens = make(B, 2, V, torch.bfloat16, seed=V)
        one = torch.ones((B, 2), device="cuda")
        _, h, lse, _, _ = atk.token_logprobs(x, tokens, top=7)
        atk.token_logprobs_grad(x, tokens, lse, h, one, one)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = atk.token_logprobs(x, tokens, top=7)
            grad = atk.token_logprobs_grad(x, tokens, out[2], out[1], one, one)
        side = torch.cuda.Stream()
        for step in range(4):
            y, _ = make(B, 2, V, torch.bfloat16, seed=step)
            x.copy_(y)
            graph.replay()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                other = atk.token_logprobs(y, tokens, top=7)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, other))
            assert torch.equal(grad, atk.token_logprobs_grad(y, tokens, other[2], other[1], one, one))
