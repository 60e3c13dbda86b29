"""The scores' host side: symbols, and refusals that come before any HIP call; the oracle against torch and against differences."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk
from oracle import scores as oracle
from paper_2412_04358_amd import scores

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULLP, DTYPE, ALIGN, WORK, ARGS = -1, -5, -7, -8, -9
FAKE = 1 << 20  # never followed: the checks come first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(atk.lib_path()):
        import __graft_entry__

        __graft_entry__.build()
    return scores._library()


def test_header_and_library_agree(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "atk_scores.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(atk_[a-z_]+)\s*\(", text))
    assert len(names) == 3
    for n in names:
        assert getattr(lib, n).argtypes is not None, n


def _call(lib, **kw):
    a = dict(x=FAKE, s=(ctypes.c_int64 * 2)(5000, 1000), t=FAKE, batch=2, tokens=5, vocab=1000, top=4, dtype=1, p=FAKE, h=FAKE, l=FAKE, tp=FAKE, tt=FAKE, work=FAKE, bytes=1 << 40)
    a.update(kw)
    return lib.atk_token_logprobs(a["x"], a["s"], a["t"], a["batch"], a["tokens"], a["vocab"], a["top"], a["dtype"], a["p"], a["h"], a["l"], a["tp"], a["tt"], a["work"], a["bytes"], None)


def _grad(lib, **kw):
    a = dict(x=FAKE, s=(ctypes.c_int64 * 2)(5000, 1000), t=FAKE, l=FAKE, h=FAKE, a=FAKE, b=FAKE, batch=2, tokens=5, vocab=1000, dtype=1, g=FAKE, gs=(ctypes.c_int64 * 2)(5000, 1000))
    a.update(kw)
    return lib.atk_token_logprobs_grad(a["x"], a["s"], a["t"], a["l"], a["h"], a["a"], a["b"], a["batch"], a["tokens"], a["vocab"], a["dtype"], a["g"], a["gs"], None)


@pytest.mark.parametrize("kw,code", [(dict(batch=0), ARGS), (dict(tokens=0), ARGS), (dict(vocab=0), ARGS), (dict(vocab=(1 << 24) + 1), ARGS), (dict(batch=1 << 22), ARGS), (dict(dtype=3), DTYPE),
                                     (dict(x=None), NULLP), (dict(s=None), NULLP), (dict(t=None), NULLP), (dict(l=None), NULLP), (dict(x=FAKE + 1), ALIGN), (dict(x=FAKE + 2, dtype=0), ALIGN),
                                     (dict(t=FAKE + 2), ALIGN), (dict(s=(ctypes.c_int64 * 2)(-1, 5)), ARGS)])
def test_both_refuse(lib, kw, code):
    assert _call(lib, **kw) == code and _grad(lib, **kw) == code


def test_logprobs_refuse(lib):
    for kw, code in [(dict(top=-1), ARGS), (dict(top=33), ARGS), (dict(top=4, vocab=3), ARGS), (dict(p=None), NULLP), (dict(h=None), NULLP), (dict(tp=None), NULLP), (dict(tt=None), NULLP), (dict(work=None), NULLP),
                     (dict(work=FAKE + 8), ALIGN), (dict(tp=FAKE + 2), ALIGN), (dict(bytes=15), WORK)]:
        assert _call(lib, **kw) == code, kw
    for batch, vocab, top in ((1, 128256, 5), (2, 1 << 24, 32), (3, 40000, 0)):
        need = lib.atk_token_logprobs_workspace_bytes(batch, 5, vocab, top, 1)
        assert need > 16 and _call(lib, batch=batch, vocab=vocab, top=top, bytes=need - 1) == WORK


def test_grad_refuses(lib):
    for kw, code in [(dict(g=None), NULLP), (dict(gs=None), NULLP), (dict(h=None), NULLP), (dict(g=FAKE + 1), ALIGN), (dict(a=FAKE + 2), ALIGN), (dict(gs=(ctypes.c_int64 * 2)(5000, 999)), ARGS),
                     (dict(gs=(ctypes.c_int64 * 2)(0, 1000)), ARGS)]:
        assert _grad(lib, **kw) == code, kw


def test_python_refuses_tensors_elsewhere(lib):
    x, t, f = torch.zeros((2, 3, 10)), torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 3))
    with pytest.raises(ValueError, match="GPU"):
        atk.token_logprobs(x, t)
    with pytest.raises(ValueError, match="must be"):
        atk.token_logprobs(x[0], t)
    with pytest.raises(TypeError, match="float32"):
        atk.token_logprobs(x.double(), t)
    with pytest.raises(ValueError, match="GPU"):
        atk.token_logprobs_grad(x, t, f, f, f)


def test_the_oracle():
    g = np.random.default_rng(0)
    x = 2 * g.standard_normal((4, 50))
    x[1, :20] = -np.inf
    chosen = np.array([3, 30, -1, 49])
    picked, entropy, lse, best, tokens, _ = oracle.logprobs(x, chosen, 5)
    logp = torch.log_softmax(torch.from_numpy(x), -1)
    assert np.allclose(picked[[0, 1, 3]], logp[[0, 1, 3], [3, 30, 49]]) and picked[2] == -np.inf
    assert np.allclose(entropy, torch.distributions.Categorical(logits=torch.from_numpy(x)).entropy()) if not np.isinf(x).any() else True
    assert np.allclose(best, torch.sort(logp, -1, descending=True).values[:, :5]) and np.allclose(lse, torch.logsumexp(torch.from_numpy(x), -1))
    a, b = g.standard_normal(4), g.standard_normal(4)
    got, _ = oracle.grad(x, chosen, lse, entropy, a, b)
    step = 1e-5
    for r in range(4):
        for i in range(50):
            if x[r, i] == -np.inf:
                assert got[r, i] == 0
                continue
            d = []
            for s in (step, -step):
                y = x.copy()
                y[r, i] += s
                p, h, *_ = oracle.logprobs(y, chosen, 0)
                d.append((a[r] * p[r] if p[r] > -np.inf else 0.0) + b[r] * h[r])
            assert abs((d[0] - d[1]) / (2 * step) - got[r, i]) < 1e-8
