"""shared_prefix_attention where many rows meet the shared keys: own keys in the same launch, in a launch of their own, past the caches, or none; against products in 64 bits on the GPU.

Tolerances as in test_gpu_decode_attention.py: h half a step of the type, e = 2^-24; weights and results are rounded to the type, scores are sums of dim products in f32, 2^x is good
to 4 e, sums over n keys add n e; f16 weights have steps of 2^-31 of the largest."""
import pytest
import torch

import paper_2412_04358_amd as atk

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
E = 2.0 ** -24


@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("B,Hk,D,prefix,ps,own", [
    (257, 128, 64, 960, 16, 16), (513, 64, 64, 950, 16, 20), (1030, 16, 96, 3000, 24, 24), (1030, 16, 128, 3001, 8, 15),  # eight wavefronts, own keys apart
    (130, 4, 128, 1024, 16, 0), (130, 4, 96, 1024, 16, 0), (70, 2, 64, 1000, 8, 0),                                       # four, no room for own keys
    (1030, 16, 128, 1600, 32, 32), (300, 8, 128, 1337, 16, 40), (300, 8, 72, 1337, 16, 40), (140, 12, 64, 1000, 4, 100),  # own keys in the same launch, the first ones past the caches
], ids=str)
@pytest.mark.parametrize("short", [False, True], ids=["all", "short"])
def test_many_rows(dtype, B, Hk, D, prefix, ps, own, short):
    g = torch.Generator(device="cuda").manual_seed(prefix + B + D)
    rest = prefix % ps                                   # tokens of the prefix in a page of each sequence's own
    shared, extra = prefix // ps, -(-(rest + own) // ps)
    P = shared + B * extra
    ids = torch.randperm(P, generator=g, device="cuda")
    table = torch.empty((B, shared + extra), dtype=torch.int64, device="cuda")
    table[:, :shared], table[:, shared:] = ids[:shared], ids[shared:].reshape(B, extra)
    room = extra * ps - rest
    lens = prefix + torch.randint(0, room + 1, (B,), generator=g, device="cuda")
    if short:  # sequences that end inside the prefix, before it, at its last key
        lens[B // 2], lens[B - 1], lens[3], lens[0] = prefix // 2, 0, prefix - 1, 1
    k, v = (torch.randn((P, ps, Hk, D), generator=g, device="cuda").to(dtype) for _ in range(2))
    at = torch.arange(room, device="cuda")
    unseen = prefix + at[None, :] >= lens[:, None]       # slots behind a sequence's last key hold NaN
    for x in (k, v):
        if rest:
            x[table[1:, shared], :rest] = x[table[0, shared], :rest].clone()
        if room:
            own_ids = table[:, shared:].repeat_interleave(ps, 1)[:, rest:]
            slots = ((rest + at) % ps).expand(B, room)
            x[own_ids[unseen], slots[unseen]] = float("nan")
    q = torch.randn((B, 1, Hk, D), generator=g, device="cuda").to(dtype)
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    out, lse = atk.shared_prefix_attention(q, k, v, table.int(), lens.int(), prefix, return_lse=True, status=status)
    assert status.item() == 0
    h, sees = HALF[dtype], torch.arange(prefix + room, device="cuda")[None, :] < lens[:, None]
    for head in range(Hk):
        kp, vp = (x[table[0], :, head].reshape(-1, D)[:prefix].double() for x in (k, v))
        ko, vo = (x[table[:, shared:], :, head].reshape(B, -1, D)[:, rest:].double().nan_to_num(0.0) for x in (k, v))
        qq = q[:, 0, head].double()

        def scores(a, kp, ko):
            return torch.cat([a @ kp.t().contiguous(), (a[:, None, :] * ko).sum(2)], 1) * D ** -0.5

        def valued(w, vp, vo):
            return w[:, :prefix].contiguous() @ vp + (w[:, prefix:, None] * vo).sum(1)

        s = scores(qq, kp, ko).masked_fill(~sees, float("-inf"))
        wlse = torch.logsumexp(s, 1)
        w = torch.exp(s - wlse[:, None]).masked_fill(~sees, 0.0)
        want, mass = valued(w, vp, vo), valued(w, vp.abs(), vo.abs())
        size = scores(qq.abs(), kp.abs(), ko.abs()).masked_fill(~sees, 0.0).amax(1)
        weight = 2 * (D + 4) * E * size + (4 + prefix + room) * E
        tol = mass * (h + 2 * weight)[:, None] + h * want.abs()
        if dtype == torch.float16:
            tol = tol + 2 * (prefix + room) * max(vp.abs().max(), vo.abs().max() if room else 0) * 2.0 ** -31 + 2.0 ** -24
        assert ((out[:, 0, head].double() - want).abs() <= tol).all()
        live = lens > 0
        assert ((lse[:, 0, head].double() - wlse)[live].abs() <= (weight + 4 * E * (1 + wlse.abs()))[live]).all()
        assert (lse[~live, 0, head] == float("-inf")).all() and (out[~live, 0, head] == 0).all()
