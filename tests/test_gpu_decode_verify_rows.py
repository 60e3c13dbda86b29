"""verify_drafts on rows at the limit of what one workgroup takes: tokens drawn from both sides of every border between its wavefronts' and chunks' shares."""
import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,most", [(torch.float32, 32768), (torch.bfloat16, 65536), (torch.float16, 65536)], ids=str)
@pytest.mark.parametrize("less", [0, 1, 513, 8192, 8195, 20000, -1])
def test_tokens_at_all_borders(dtype, most, less):
    V = most - less
    # equal weights, a power of two: sums are exact, and the token is the whole part of r * V; rows of 512 elements to a chunk and fewer to a wavefront's share
    at = np.unique(np.clip(np.concatenate([np.arange(0, V + 512, 512) + d for d in (-1, 0, 1)] + [np.array([0, V - 1])]), 0, V - 1))
    r = torch.from_numpy(((at + 0.5) / V).astype(np.float32)).clamp(max=1 - 2.0 ** -24)
    want = np.floor(r.double().numpy() * V).astype(np.int64)
    assert (want == at).all()     # (r's rounding, V * 2^-25, is far below 0.5)
    n = len(at)
    target = torch.full((V,), 2.0 ** -14, dtype=dtype, device="cuda").expand(n, 1, V)     # one row for all
    none = torch.zeros((n, 0), device="cuda")
    accepted, tokens = atk.verify_drafts(target, none.int(), None, none, r.cuda())
    assert (accepted == 0).all() and np.array_equal(tokens[:, 0].cpu().numpy(), want)
    # the same behind a rejection: twice the weight less the draft's
    u = torch.full((n, 1), 0.9, device="cuda")
    first = torch.full((n, 1), V // 2, dtype=torch.int32, device="cuda")
    two = torch.full((V,), 2.0 ** -13, dtype=dtype, device="cuda")
    low = two.clone()
    low[V // 2] = 0.0                                          # (the drafted token: never accepted, no weight)
    draft = torch.full((V,), 2.0 ** -14, dtype=dtype, device="cuda").expand(n, 1, V)
    accepted, tokens = atk.verify_drafts(torch.stack([low, two]).expand(n, 2, V), first, draft, u, r.cuda())
    goal = r.double().numpy() * (V - 1)
    index = np.floor(goal).astype(np.int64)
    sure = np.abs(goal - np.round(goal)) > 1e-6
    index = index + (index >= V // 2)
    assert (accepted == 0).all() and np.array_equal(tokens[:, 0].cpu().numpy()[sure], index[sure]) and (tokens[:, 1] == -1).all()
