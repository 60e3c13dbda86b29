"""The cache's calls on lengths and counts at the ends of 32 bits: reported or refused, and nothing done."""
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("page_size", [16, 24, 65537, (1 << 20) + 1])
@pytest.mark.parametrize("length", [(1 << 31) - 1, (1 << 31) - 65536, (1 << 30) + 1, -1, -(1 << 31)])
def test_fork_from_a_length_that_no_row_holds(page_size, length):
    t = atk.PageTables.empty(6, page_size, 4, 3)
    pool = torch.zeros((6, page_size, 1), dtype=torch.uint8, device="cuda")
    t.lens[1] = length
    before = [x.clone() for x in (t.page_table, t.lens, t.refs, t.free_pages, t.n_free)]
    atk.fork_sequences(t, [pool], ints([1]), ints([2]))
    torch.cuda.synchronize()
    assert t.status.item() == atk.ATK_STATUS_BAD_LEN
    assert all(torch.equal(a, b) for a, b in zip(before, (t.page_table, t.lens, t.refs, t.free_pages, t.n_free))) and not pool.any()
