"""verify_drafts against its definition: whole numbers, so equal - the random numbers' distance from a border is checked to be far above what 64-bit sums are off by."""
import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk
from oracle import decode as oracle

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def make(B, L, V, dtype, seed, agree=0.7, pad=0):
    g = torch.Generator().manual_seed(seed)
    logits = 3 * torch.randn((B, L + 1, V), generator=g)
    target = torch.softmax(logits, -1)
    draft = torch.softmax(logits[:, :L] + agree * torch.randn((B, L, V), generator=g), -1)
    tokens = torch.multinomial(draft.reshape(B * L, V), 1, generator=g).reshape(B, L).int() if L else torch.zeros((B, 0), dtype=torch.int32)
    wide_t, wide_d = torch.full((B, L + 1, V + pad), 9.0, dtype=dtype), torch.full((B, L, V + pad), 9.0, dtype=dtype)
    wide_t[..., :V], wide_d[..., :V] = target.to(dtype), draft.to(dtype)
    return [wide_t.cuda()[..., :V], tokens.cuda(), wide_d.cuda()[..., :V], torch.rand((B, L), generator=g).cuda(), torch.rand((B,), generator=g).cuda()]


def check(target, tokens, draft, u, r, n_drafts=None):
    accepted, out = atk.verify_drafts(target, tokens, draft, u, r, n_drafts=n_drafts)
    torch.cuda.synchronize()
    host = [None if x is None else x.double().cpu().numpy() if x.is_floating_point() else x.cpu().numpy() for x in (target, tokens, draft, u, r, n_drafts)]
    want, wout, near = oracle.verify(*host)
    # a sum of V numbers in 64 bits is off by V * 2^-53 of the total at most
    assert near.min() > target.shape[2] * 2.0 ** -53 or not np.isfinite(near).any()
    assert np.array_equal(accepted.cpu().numpy(), want) and np.array_equal(out.cpu().numpy(), wout)
    return accepted, out


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("B,L,V,pad", [(1, 1, 1, 0), (1, 4, 2, 0), (3, 2, 63, 1), (2, 5, 1000, 0), (7, 3, 2049, 7), (4, 8, 32000, 0), (64, 2, 5003, 5), (2, 100, 700, 0), (1, 3, 50257, 0), (300, 1, 4100, 0),
                                       (3, 2, 128256, 64)])
def test_shapes(dtype, B, L, V, pad):
    accepted, _ = check(*make(B, L, V, dtype, seed=V + L, pad=pad))
    if B * L > 100:
        assert 0 < accepted.float().mean() < L


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("V", [3001, 70001])   # rows by one workgroup, rows by many
def test_no_drafts_and_ragged_drafts(dtype, V):
    target, tokens, draft, u, r = make(6, 4, V, dtype, seed=5, agree=0.1)
    check(target, tokens, draft, u, r, torch.tensor([0, 1, 2, 3, 4, 9], dtype=torch.int32, device="cuda"))
    check(target, tokens, draft, u, r, torch.tensor([-3, 1, 0, 0, 4, 4], dtype=torch.int32, device="cuda"))
    args = make(3, 0, V, dtype, seed=6)
    accepted, out = check(*args)
    assert (accepted == 0).all() and out.shape == (3, 1)
    check(args[0], args[1], None, args[3], args[4])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("V", [37, 66003])
def test_certain_drafts(dtype, V):
    target, tokens, _, u, r = make(40, 4, 37, dtype, seed=7)
    wide = torch.zeros((40, 5, V), dtype=dtype, device="cuda")
    wide[..., V - 37:] = target
    target = wide
    tokens = target[:, :4].float().argmax(2).int()
    accepted, out = check(target, tokens, None, u, r)
    rejected = accepted < 4
    rows = torch.arange(40, device="cuda")
    assert rejected.any() and (out[rows, accepted.long()][rejected] != tokens[rows, accepted.clamp(max=3).long()][rejected]).all()


def test_borders():
    # u * q == p is a rejection, the next smaller u is not; sums that meet the goal exactly go to the next index
    target = torch.tensor([[[0.25, 0.25, 0.5], [0.5, 0.25, 0.25]]], device="cuda")
    draft = torch.tensor([[[0.5, 0.25, 0.25]]], device="cuda")
    tokens = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    half = torch.tensor([[0.5]], device="cuda")
    for u, want in ((half, 0), (torch.nextafter(half, torch.zeros_like(half)), 1)):
        for r, token in ((0.0, 0), (0.25, 0), (0.5, 1), (0.75, 2), (1 - 2 ** -24, 2)):
            accepted, out = atk.verify_drafts(target, tokens, draft, u, torch.tensor([r], device="cuda"))
            assert accepted.item() == want
            assert out.tolist() == [[2, -1]] if want == 0 else [[0, token]]


@pytest.mark.parametrize("V", [300, 70000])
def test_weights_of_nothing(V):
    z = torch.zeros((2, 2, V), device="cuda")
    u, r = torch.full((2, 1), 0.5, device="cuda"), torch.tensor([0.0, 0.9], device="cuda")
    tokens = torch.tensor([[5], [V - 1]], dtype=torch.int32, device="cuda")
    accepted, out = check(z, tokens, z[:, :1], u, r)                      # no weight anywhere: no token
    assert (accepted == 0).all() and (out == -1).all()
    p = z.clone()
    p[:, :, 7], p[:, :, 250] = 0.5, 0.5
    accepted, out = check(p, tokens, p[:, :1], u, r)                      # rejected (p is 0 there) with nothing left: p itself
    assert out[:, 0].tolist() == [7, 250]
    accepted, out = check(p, torch.tensor([[-1], [V]], dtype=torch.int32, device="cuda"), z[:, :1], u, r)   # tokens outside the vocabulary
    assert (accepted == 0).all() and out[:, 0].tolist() == [7, 250]
    p[:, :, 8], p[:, :, 100] = float("nan"), -0.25                        # weigh nothing
    accepted, out = atk.verify_drafts(p, tokens, z[:, :1], u, r)
    assert out[:, 0].tolist() == [7, 250]
    p[:, :, 9] = float("inf")                                             # no sum: some index, none out of range
    _, out = atk.verify_drafts(p, tokens, z[:, :1], u, r)
    assert ((out[:, 0] >= -1) & (out[:, 0] < V)).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_ends_of_the_running_sum(dtype):
    # single weights at the first and last element, equal weights (exact sums), r from 0 to the largest below 1
    for V in (257, 4096, 20001, 32768, 66001, 133000):
        p = torch.zeros((4, 1, V), dtype=dtype)
        p[0, 0, 0] = p[1, 0, V - 1] = 1.0
        p[2, 0, :] = 2.0 ** -12
        p[3, 0, ::2] = 2.0 ** -12
        none = torch.zeros((4, 0), dtype=torch.int32, device="cuda")
        for r in (0.0, 0.5 + 2.0 ** -20, 1 - 2.0 ** -24):
            rr = torch.full((4,), r, device="cuda")
            accepted, out = atk.verify_drafts(p.cuda(), none, None, torch.zeros((4, 0), device="cuda"), rr)
            want = oracle.verify(p.double().numpy(), none.cpu().numpy(), None, np.zeros((4, 0)), rr.cpu().numpy())[1]
            assert np.array_equal(out.cpu().numpy(), want)


@pytest.mark.parametrize("V", [32001, 90001])
def test_streams_and_graph(V):
    args = make(8, 4, V, torch.bfloat16, seed=21)
    want = check(*args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = atk.verify_drafts(*args)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = atk.verify_drafts(*args)
    for step in range(4):
        args[4].copy_(torch.rand((8,), generator=torch.Generator().manual_seed(step)))
        want = atk.verify_drafts(*args)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), step


def test_refusals():
    target, tokens, draft, u, r = make(2, 3, 100, torch.float32, seed=1)
    with pytest.raises(ValueError, match="target_probs must"):
        atk.verify_drafts(target[:, :3], tokens, draft, u, r)
    with pytest.raises(TypeError, match="int32"):
        atk.verify_drafts(target, tokens.long(), draft, u, r)
    with pytest.raises(TypeError, match="type"):
        atk.verify_drafts(target, tokens, draft.half(), u, r)
    with pytest.raises(ValueError, match="contiguous"):
        atk.verify_drafts(target.transpose(1, 2).contiguous().transpose(1, 2), tokens, draft, u, r)
    with pytest.raises(TypeError, match="float32"):
        atk.verify_drafts(target, tokens, draft, u.double(), r)
    with pytest.raises(ValueError, match="shape"):
        atk.verify_drafts(target, tokens, draft, u, r[:1])
    with pytest.raises(ValueError, match="GPU"):
        atk.verify_drafts(target, tokens.cpu(), draft, u, r)
    assert [tuple(t.shape) for t in atk.verify_drafts(target[:0], tokens[:0], draft[:0], u[:0], r[:0])] == [(0,), (0, 4)]
