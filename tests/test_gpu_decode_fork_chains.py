"""fork_sequences where a parent is a child of the same call: a row is forked as it is at the call, and children are empty there."""
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("n", [2, 65, 130, 257, 700])
@pytest.mark.parametrize("order", ["chain", "last", "shuffled"])
def test_children_that_are_parents(n, order):
    ps, rows = 4, n + 1
    t = atk.PageTables.empty(8 + n, ps, rows, 4)
    pool = torch.zeros((8 + n, ps, 3), device="cuda")
    value = torch.arange(1, 1 + 6 * 3, device="cuda").float().reshape(1, 6, 3)
    atk.append_tokens(t, [pool], ints([0]), [value])            # row 0: a whole page and a part of one
    children = list(range(1, n + 1))
    if order == "chain":
        parents = list(range(n))                                # each row the next one's parent
    else:
        parents = [0] + [1] * (n - 1)                           # row 0 -> 1, and 1, empty at the call, -> all others
    if order == "shuffled":
        perm = torch.randperm(n, generator=torch.Generator().manual_seed(n)).tolist()
        parents, children = [parents[i] for i in perm], [children[i] for i in perm]
    atk.fork_sequences(t, [pool], ints(parents), ints(children))
    torch.cuda.synchronize()
    assert t.status.item() == 0
    assert t.lens.tolist() == [6, 6] + [0] * (n - 1)
    assert t.page_table.tolist() == [[0, 1, -1, -1], [0, 2, -1, -1]] + [[-1] * 4] * (n - 1)
    assert t.refs.tolist() == [2, 1, 1] + [0] * (5 + n) and t.n_free.item() == 5 + n
    assert torch.equal(pool[2, :2], value[0, 4:])


def test_a_row_that_is_its_own_parent():
    t = atk.PageTables.empty(4, 4, 3, 2)
    pool = torch.zeros((4, 4, 1), device="cuda")
    atk.fork_sequences(t, [pool], ints([1, 1]), ints([1, 2]))
    torch.cuda.synchronize()
    assert t.status.item() == 0 and t.lens.tolist() == [0, 0, 0] and (t.page_table == -1).all() and t.n_free.item() == 4
    # one that holds something is no child
    atk.append_tokens(t, [pool], ints([1]), [torch.ones((1, 3, 1), device="cuda")])
    atk.fork_sequences(t, [pool], ints([1]), ints([1]))
    torch.cuda.synchronize()
    assert t.status.item() == atk.ATK_STATUS_BAD_SEQ and t.lens.tolist() == [0, 3, 0]
