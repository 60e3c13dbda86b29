"""Plain definition of the scores of tokens in 64 bits (test infrastructure only)."""
from __future__ import annotations

import numpy as np


def logprobs(x, chosen, top):
    """x (rows, vocab) f64 -> logprobs, entropy, lse (rows), top_logprobs, top_tokens (rows, top), and per row the mean of |log p|."""
    rows, V = x.shape
    lse, entropy, picked, mean = np.full(rows, -np.inf), np.zeros(rows), np.full(rows, -np.inf), np.zeros(rows)
    best, tokens = np.full((rows, top), -np.inf), np.zeros((rows, top), np.int64)
    for r in range(rows):
        order = sorted(range(V), key=lambda i: (-(x[r, i] if x[r, i] == x[r, i] else -np.inf), i))[:top]
        tokens[r] = order
        if not np.all(x[r] < np.inf):      # a NaN or +inf
            lse[r] = entropy[r] = np.nan
            picked[r] = np.nan if 0 <= chosen[r] < V else -np.inf
            best[r] = np.nan
            continue
        m = x[r].max()
        if m == -np.inf:
            continue
        lse[r] = m + np.log(np.exp(x[r] - m).sum())
        logp = x[r] - lse[r]
        p = np.exp(logp)
        entropy[r] = -(p[p > 0] * logp[p > 0]).sum()
        mean[r] = (p[p > 0] * np.abs(logp[p > 0])).sum()
        best[r] = logp[order]
        if 0 <= chosen[r] < V:
            picked[r] = logp[chosen[r]]
    return picked, entropy, lse, best, tokens, mean


def grad(x, chosen, lse, entropy, a, b):
    """Gradient (rows, vocab) from the formula, and what its terms' sizes add up to."""
    rows, V = x.shape
    out, size = np.zeros((rows, V)), np.zeros((rows, V))
    for r in range(rows):
        if lse[r] == -np.inf:
            continue
        with np.errstate(invalid="ignore"):
            logp = x[r] - lse[r]
        p = np.exp(logp)
        ar = a[r] if 0 <= chosen[r] < V else 0.0
        some = p > 0
        out[r, some] = -p[some] * (ar + b[r] * (logp[some] + entropy[r]))
        out[r, np.isnan(p)] = np.nan
        size[r, some] = p[some] * (abs(ar) + abs(b[r]) * (np.abs(logp[some]) + abs(entropy[r])))
        if 0 <= chosen[r] < V:
            out[r, chosen[r]] += ar
            size[r, chosen[r]] += abs(ar)
    return out, size
