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
