"""token_logprobs on rows that lie far from 0: all of the type's lowest or largest value, or ordinary ones moved by more than the type's whole numbers resolve of a log.

Against the definition in 64 bits from the rows' largest logit m, x - m - log sum e^(x - m): from log sum e^x it would be lost in 64 bits too.  The tolerance is that of the other tests of scores but for what
an lse of size costs: with e = 2^-24, delta = (24 + 3 (mean + 4) + chain) e for the sum, log p the difference of x - r (r within 4 of m), good to e of itself, and log Z, to delta and 2 e of itself."""
import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
E = 2.0 ** -24


def definition(x):
    """log p, entropy, the mean of |log p|, of rows (n, vocab) f64."""
    d = x - x.max(1, keepdims=True)
    logp = d - np.log(np.exp(d).sum(1, keepdims=True))
    p = np.exp(logp)
    mean = np.where(p > 0, p * np.abs(np.where(p > 0, logp, 0)), 0).sum(1)
    return logp, mean, mean


def make(kind, B, V, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    info = torch.finfo(dtype)
    if kind == "lowest":
        x = torch.full((B, 1, V), info.min, dtype=dtype)
    elif kind == "largest":
        x = torch.full((B, 1, V), info.max, dtype=dtype)
    elif kind == "lowest but for -inf":
        x = torch.full((B, 1, V), info.min, dtype=dtype)
        x[torch.rand((B, 1, V), generator=g) < 0.5] = -float("inf")
        x[..., V // 3] = info.min
    else:   # steps of the type that are coarse, but not against what the logits differ by
        shift = {"above": 1.0, "below": -1.0}[kind] * (2.0 ** 14 if dtype is torch.float32 else 2.0 ** 11)
        x = (3 * torch.randn((B, 1, V), generator=g, dtype=torch.float64) + shift).to(dtype)
    return x.cuda()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("kind", ["lowest", "largest", "lowest but for -inf", "above", "below"])
@pytest.mark.parametrize("B,V,top", [(1, 1, 1), (2, 300, 5), (1, 32000, 20), (2, 40000, 9), (3, 40000, 0), (260, 5000, 0), (1, 270000, 32)])
def test_far_rows(dtype, kind, B, V, top):
    x = make(kind, B, V, dtype, seed=V)
    tokens = torch.full((B, 1), V // 3, dtype=torch.int32, device="cuda")
    got, entropy, lse, best, order = [t.double().cpu().numpy()[:, 0] for t in atk.token_logprobs(x, tokens, top=top)]
    some = sorted({0, B // 2, B - 1})
    rows = x[some, 0].double().cpu().numpy()
    logp, want_h, mean = definition(rows)
    delta = (24 + 3 * (mean + 4) + 2 * V / 256 + 8) * E
    log_z = np.log(V) + 4
    off = delta + 2 * E * log_z
    picked = logp[:, V // 3]
    assert (np.abs(got[some] - picked) <= off + 3 * E * (np.abs(picked) + log_z)).all()
    assert (np.abs(entropy[some] - want_h) <= off + (2 * delta + 4 * E) * (mean + 8)).all()
    for i, r in enumerate(some):
        first = np.lexsort((np.arange(V), -rows[i]))[:top]
        assert np.array_equal(order[r], first)
        want = logp[i, first]
        fine = np.isfinite(want)
        assert np.array_equal(best[r][~fine], want[~fine])
        assert (np.abs(best[r] - want)[fine] <= (off[i] + 3 * E * (np.abs(want) + log_z))[fine]).all()
        assert abs(lse[r] - (rows[i].max() + np.log(np.exp(rows[i] - rows[i].max()).sum()))) <= off[i] + 2 * E * abs(rows[i].max()) + E * abs(lse[r])
