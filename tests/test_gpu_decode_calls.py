"""The decoding operators' calls on plain tensors, which an extension module marshals, against the same calls marshalled by decode.py; and an end to end loop of all of them."""
import pytest
import torch

import paper_2412_04358_amd as atk
from paper_2412_04358_amd import decode

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.fixture
def by_python(monkeypatch):
    """Calls the function a second time with the module switched off."""
    decode._load_plain()
    assert decode._plain

    def both(f):
        first = f()
        monkeypatch.setattr(decode, "_plain", False)
        second = f()
        monkeypatch.undo()
        return first, second

    return both


def same(a, b):
    assert type(a) is type(b)
    for x, y in zip(a, b) if isinstance(a, tuple) else [(a, b)]:
        assert type(x) is type(y) is torch.Tensor and x.dtype == y.dtype and x.shape == y.shape and x.device == y.device and torch.equal(x, y)


def test_attention_and_verification(by_python):
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((40, 16, 2, 64), generator=g, device="cuda").half() for _ in range(2))
    q = torch.randn((5, 2, 8, 64), generator=g, device="cuda").half()
    table = torch.arange(40, device="cuda").int().reshape(5, 8)
    lens = ints([100, 60, 77, 128, 3])
    for lse in (True, False):
        for seqs in (None, ints([3, 1, 0, 2, 4])):
            for scale in (None, 0.3):
                same(*by_python(lambda: atk.shared_prefix_attention(q, k, v, table, lens, 20, seqs=seqs, scale=scale, return_lse=lse)))
    p = torch.softmax(3 * torch.randn((4, 4, 999), generator=g, device="cuda"), -1)
    d = torch.softmax(torch.randn((4, 3, 999), generator=g, device="cuda"), -1)
    tokens, u, r = torch.randint(0, 999, (4, 3), generator=g, device="cuda").int(), torch.rand((4, 3), generator=g, device="cuda"), torch.rand((4,), generator=g, device="cuda")
    for n in (None, ints([0, 1, 2, 3])):
        for draft in (d, None):
            same(*by_python(lambda: atk.verify_drafts(p, tokens, draft, u, r, n_drafts=n)))
    # what is no plain tensor
    class Sub(torch.Tensor):
        pass

    assert torch.equal(atk.verify_drafts(p.as_subclass(Sub), tokens, d, u, r)[1].as_subclass(torch.Tensor), atk.verify_drafts(p, tokens, d, u, r)[1])


def test_pages(by_python):
    def life():
        t = atk.PageTables.empty(30, 4, 6, 6)
        pools = [torch.zeros((30, 4, 3), device="cuda") for _ in range(2)]
        values = [torch.arange(2 * 5 * 3, device="cuda").float().reshape(2, 5, 3) + i for i in range(2)]
        atk.append_tokens(t, pools, ints([0, 2]), values)
        atk.fork_sequences(t, pools, ints([0, 2]), ints([1, 5]))
        atk.append_tokens(t, pools, ints([1, 0]), values)
        atk.free_sequences(t, ints([0, 1]), drop=ints([1, 7]))
        atk.free_sequences(t, ints([2]))
        remap = atk.compact_pages(t, pools)
        other = [torch.zeros_like(p) for p in pools]
        atk.copy_pages(pools, ints([0, 3]), other, ints([7, 1]))
        return (t.page_table, t.lens, t.refs, t.free_pages, t.n_free, t.status, remap, *pools, *other)

    first, second = by_python(life)
    same(first, second)
    assert first[5].item() == 0


def test_decoding_loop_is_decoding():
    """Samples of one prompt with drafts, against the same steps without a cache: examples/decode_samples.py."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_samples.py")
    spec = importlib.util.spec_from_file_location("decode_samples", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    report = m.run(samples=5, prompt=83, steps=6, drafts=3, check=True, quiet=True)
    assert report["tokens"] >= 5 * 6 and 0 <= report["accepted"] <= 1 and report["worst"] < 1.0
