"""copy_pages on caches without pages or without tokens: refused, and nothing else happens; without anything to copy it is nothing."""
import pytest
import torch

import paper_2412_04358_amd as atk
from paper_2412_04358_amd import decode

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("by_module", [True, False])
def test_caches_that_hold_nothing(by_module, monkeypatch):
    if not by_module:
        monkeypatch.setattr(decode, "_plain", False)

    def pool(*shape):
        return [torch.zeros(shape, device="cuda")]

    for src, dst in ((pool(0, 16, 4), pool(3, 16, 4)), (pool(3, 16, 4), pool(0, 16, 4)), (pool(0, 16, 4), pool(0, 16, 4)), (pool(3, 0, 4), pool(3, 0, 4))):
        with pytest.raises(ValueError, match="a page, and a token"):
            atk.copy_pages(src, ints([0]), dst, ints([1]))
        atk.copy_pages(src, ints([]), dst, ints([]))


def test_tokens_of_no_bytes():
    # a view of no elements has its tensor's address
    whole = torch.arange(6 * 4 * 2, device="cuda").float().reshape(6, 4, 2)
    kept = whole.clone()
    none = [whole[:, :, :0]]
    t = atk.PageTables.empty(6, 4, 3, 2)
    for call in (lambda: atk.copy_pages(none, ints([0]), none, ints([1])), lambda: atk.append_tokens(t, none, ints([0]), [torch.zeros((1, 5, 0), device="cuda")]),
                 lambda: atk.fork_sequences(t, none, ints([0]), ints([1])), lambda: atk.compact_pages(t, none)):
        with pytest.raises(ValueError, match="a byte for a token"):
            call()
    torch.cuda.synchronize()
    assert torch.equal(whole, kept) and t.lens.tolist() == [0, 0, 0] and t.status.item() == 0
    # no pools at all are tables alone
    atk.fork_sequences(t, [], ints([0]), ints([1]))
    assert (atk.compact_pages(t, []) == -1).all()
