"""The calls of quantized.py and scores.py on plain tensors, which an extension module marshals, against the same calls marshalled in Python; and a run of them together."""
import pytest
import torch

import paper_2412_04358_amd as atk
from oracle import decode as plain_attention
from oracle import quant as oracle
from oracle import scores as plain_scores
from paper_2412_04358_amd import plain

pytestmark = pytest.mark.gpu


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.fixture
def by_python(monkeypatch):
    """Calls the function a second time with the module switched off."""
    assert plain._load()

    def both(f):
        first = f()
        monkeypatch.setattr(plain, "_module", False)
        second = f()
        monkeypatch.undo()
        return first, second

    return both


def same(a, b):
    assert type(a) is type(b)
    for x, y in zip(a, b) if isinstance(a, (tuple, list)) else [(a, b)]:
        assert type(x) is type(y) is torch.Tensor and x.dtype == y.dtype and x.shape == y.shape and x.device == y.device and torch.equal(x, y)


def test_attention(by_python):
    g = torch.Generator(device="cuda").manual_seed(1)
    pools = [torch.randint(100, 130, (40, 16, atk.quantized_token_bytes(2, 64)), generator=g, device="cuda").to(torch.uint8) for _ in range(2)]
    q = torch.randn((5, 2, 8, 64), generator=g, device="cuda").half()
    table = torch.arange(40, device="cuda").int().reshape(5, 8)
    lens = ints(100, 60, 77, 128, 3)
    for lse in (True, False):
        for seqs in (None, ints(3, 1, 0, 2, 4)):
            for scale in (None, 0.3, 1):
                for status in (None, ints(0)):
                    same(*by_python(lambda: atk.quantized_attention(q, *pools, table, lens, 2, seqs=seqs, scale=scale, return_lse=lse, status=status)))


def test_pages(by_python):
    g = torch.Generator(device="cuda").manual_seed(1)
    values = [torch.randn((2, 5, 3, 32), generator=g, device="cuda").bfloat16() for _ in range(2)]

    def life():
        t = atk.PageTables.empty(30, 4, 6, 6)
        pools = [torch.zeros((30, 4, atk.quantized_token_bytes(3, 32, 8)), dtype=torch.uint8, device="cuda") for _ in range(2)]
        atk.append_quantized(t, pools, ints(0, 2), values, bits=8)
        atk.fork_sequences(t, pools, ints(0, 2), ints(1, 5))
        atk.append_quantized(t, pools, ints(1, 0), tuple(values), bits=8)
        out = [atk.read_quantized(t, pools, ints(0, 1, 5), starts, 7, 3, 32, bits=8, dtype=dtype) for starts in (None, ints(3, 0, 9)) for dtype in (None, torch.float32, torch.float16)]
        return (t.page_table, t.lens, t.refs, t.n_free, t.status, *pools, *(x for pair in out for x in pair))

    first, second = by_python(life)
    same(first, second)
    assert first[4].item() == 0


def test_scores(by_python):
    g = torch.Generator(device="cuda").manual_seed(1)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn((3, 2, 999), generator=g, device="cuda").to(dtype)[:, :, 1:]
        tokens = torch.randint(0, 998, (3, 2), generator=g, device="cuda").int()
        for top in (0, 4):
            first, second = by_python(lambda: atk.token_logprobs(x, tokens, top=top))
            same(first, second)
        a, b = torch.randn((3, 2), generator=g, device="cuda"), torch.randn((3, 2), generator=g, device="cuda")
        for args in ((a, b), (a,), (None, b)):
            same(*by_python(lambda: atk.token_logprobs_grad(x, tokens, first[2], first[1], *args)))

    # what is no plain tensor
    class Sub(torch.Tensor):
        pass

    assert torch.equal(atk.token_logprobs(x.as_subclass(Sub), tokens)[0].as_subclass(torch.Tensor), atk.token_logprobs(x, tokens)[0])


@pytest.mark.parametrize("bits", [4, 8])
def test_samples_are_decoded_and_scored(bits):
    """A prompt goes into the cache, is forked, samples grow with drafts that are partly dropped, their tokens are scored, and a gradient follows; all of it against plain definitions."""
    import numpy as np

    heads, kv, dim, vocab, ps, B = 8, 2, 64, 500, 16, 3
    g = torch.Generator().manual_seed(5)
    head = (torch.randn((heads * dim, vocab), generator=g) * 0.3).cuda()
    t = atk.PageTables.empty(60, ps, B + 1, 12)
    pools = [torch.zeros((60, ps, atk.quantized_token_bytes(kv, dim, bits)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    prompt = [torch.randn((1, 37, kv, dim), generator=g).bfloat16() for _ in range(2)]
    atk.append_quantized(t, pools, ints(0), [x.cuda() for x in prompt], bits=bits)
    rows = ints(1, 2, 3)
    atk.fork_sequences(t, pools, ints(0, 0, 0), rows)
    kept = [[[x[0]] for x in prompt] for _ in range(B)]
    for step in range(4):
        new = [torch.randn((B, 3, kv, dim), generator=g).bfloat16() for _ in range(2)]
        atk.append_quantized(t, pools, rows, [x.cuda() for x in new], bits=bits)
        q = torch.randn((B, 3, heads, dim), generator=g).bfloat16()
        out = atk.quantized_attention(q.cuda(), *pools, t.page_table, t.lens, kv, bits=bits, seqs=rows, status=t.status)
        logits = (out.float().flatten(2) @ head)
        tokens = torch.randint(0, vocab, (B, 3), generator=g).int()
        logprobs, entropy, lse, top_logprobs, top_tokens = atk.token_logprobs(logits, tokens.cuda(), top=3)
        grad = atk.token_logprobs_grad(logits, tokens.cuda(), lse, entropy, torch.ones_like(logprobs), 0.1 * torch.ones_like(entropy))
        drop = ints(*[(step + b) % 3 for b in range(B)])
        # the plain way
        for b in range(B):
            for p in range(2):
                kept[b][p].append(new[p][b])
        longest = max(sum(x.shape[0] for x in kept[b][0]) for b in range(B))
        kv_all = [np.zeros((B, longest, kv, dim)) for _ in range(2)]
        for b in range(B):
            for p in range(2):
                x = torch.cat(kept[b][p]).double().numpy()
                kv_all[p][b, :x.shape[0]] = oracle.decode(oracle.encode(x, bits), kv, dim, bits)
        lens = np.array([sum(x.shape[0] for x in kept[b][0]) for b in range(B)])
        want, _, mass, size, count, _ = plain_attention.attention(q.double().numpy(), *kv_all, np.arange(B)[:, None], lens, 0, None, dim ** -0.5)
        tol = mass * (2.0 ** -8 + 2 * (2 * (dim + 4) * 2.0 ** -24 * size + (4 + count) * 2.0 ** -24))[..., None] + 2.0 ** -8 * np.abs(want)   # as in the test of the attention
        assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
        x = logits.double().cpu().numpy().reshape(-1, vocab)
        picked, h, ll, best, order, _ = plain_scores.logprobs(x, tokens.numpy().reshape(-1), 3)
        for a, b in ((logprobs, picked), (entropy, h), (lse, ll), (top_logprobs, best)):
            assert np.abs(a.double().cpu().numpy().reshape(b.shape) - b).max() < 2.0 ** -16
        assert np.array_equal(top_tokens.cpu().numpy().reshape(order.shape), order)
        full, _ = plain_scores.grad(x, tokens.numpy().reshape(-1), ll, h, np.ones(B * 3), 0.1 * np.ones(B * 3))
        assert np.abs(grad.double().cpu().numpy().reshape(full.shape) - full).max() < 2.0 ** -16
        atk.free_sequences(t, rows, drop=drop)
        for b in range(B):
            n = int(drop[b])
            for p in range(2):
                if n:
                    kept[b][p][-1] = kept[b][p][-1][:-n]
        atk.compact_pages(t, pools)
    assert t.status.item() == 0
    assert torch.equal(atk.read_quantized(t, pools, ints(0), None, 37, kv, dim, bits=bits)[1][0].cpu().double(),
                       torch.from_numpy(oracle.decode(oracle.encode(prompt[1][0].double().numpy(), bits), kv, dim, bits)))
