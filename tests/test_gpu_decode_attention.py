"""shared_prefix_attention against its definition in 64 bits: types, head layouts, lengths from nothing on, pages that end anywhere, masks, strides.

The tolerance counts roundings, with h half a step of the type (relative) and e = 2^-24: every weight is rounded to the type (h, against the sum of weight * |v|), so is the
result (h of it); a score is a sum of dim products in f32, off by (dim + 4) e of scale * sum |q k|, and a weight by as much relatively, in the sum of weights too;
2^x is good to 4 e; sums over n keys add n e.  f16 weights have steps of 2^-32 of the largest at the least (2^-24 behind a factor of 2^8 to 2^15... taken as 2^-31)."""
import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk
from oracle import decode as oracle

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.bfloat16, torch.float16, torch.float32]
E = 2.0 ** -24


def make(B, T, H, Hk, D, prefix, lens, ps, dtype, seed=0, head_major=False, spare=2, rows=None, scale_q=1.0):
    """q, k, v, table, lens on the GPU; unused pages, unused slots and entries hold what must not matter."""
    g = torch.Generator().manual_seed(seed)
    rows = B if rows is None else rows
    M = max(1, max(-(-n // ps) for n in lens) + spare)
    shared = prefix // ps
    P = shared + rows * M + 1
    ids = torch.randperm(P, generator=g)
    table = torch.empty((rows, M), dtype=torch.int64)
    table[:, :shared] = ids[:shared]
    table[:, shared:] = ids[shared:shared + rows * (M - shared)].reshape(rows, M - shared)
    kv = []
    for _ in range(2):
        x = torch.randn((P, ps, Hk, D), generator=g).to(dtype)
        left = prefix - shared * ps
        if left:
            x[table[:, shared], :left] = x[table[0, shared], :left].clone()
        kv.append(x)
    # slots that no sequence fills hold NaN
    filled = torch.zeros((P, ps), dtype=torch.bool)
    for r in range(rows):
        for j in range(max(lens[r], prefix if r == 0 else 0)):
            filled[table[r, j // ps], j % ps] = True
    for x in kv:
        x[~filled] = float("nan")
    for r in range(rows):
        held = -(-max(lens[r], prefix) // ps)
        table[r, held:] = -1
    q = (scale_q * torch.randn((B, T, H, D), generator=g)).to(dtype)
    dev = [q.cuda(), kv[0].cuda(), kv[1].cuda()]
    if head_major:
        dev[1:] = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in dev[1:]]
    return dev + [table.int().cuda(), torch.tensor(lens, dtype=torch.int32).cuda()]


def wider(table, ps, keys=2048):
    """The table with room for more pages: sequences that could be long have their shared keys taken apart from their own."""
    wide = torch.full((table.shape[0], table.shape[1] + keys // ps), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    return wide


def check(q, k, v, table, lens, prefix, seqs=None, scale=None):
    got = _check(q, k, v, table, lens, prefix, seqs, scale)
    _check(q, k, v, wider(table, k.shape[1]), lens, prefix, seqs, scale)
    return got


def _check(q, k, v, table, lens, prefix, seqs, scale):
    D = q.shape[3]
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    out, lse = atk.shared_prefix_attention(q, k, v, table, lens, prefix, seqs=seqs, scale=scale, return_lse=True, status=status)
    torch.cuda.synchronize()
    c = [x.double().cpu().numpy() for x in (q, k, v)]
    want, wlse, mass, size, count, top = oracle.attention(*c, table.cpu().numpy(), lens.cpu().numpy(), prefix, None if seqs is None else seqs.cpu().numpy(), D ** -0.5 if scale is None else scale)
    h = HALF[q.dtype]
    weight = 2 * (D + 4) * E * size + (4 + count) * E     # relative, of a weight or of their sum
    tol = mass * (h + 2 * weight)[..., None] + h * np.abs(want)
    if q.dtype == torch.float16:
        tol = tol + 2 * (count * top * 2.0 ** -31)[..., None] + 2.0 ** -24  # (and outputs have subnormal steps)
    got_out, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert status.item() == 0
    assert np.array_equal(np.isnan(got_out), np.isnan(want)) and np.array_equal(np.isnan(got_lse), np.isnan(wlse))
    finite = np.isfinite(want)
    assert (np.abs(got_out - want)[finite] <= tol[finite]).all(), np.nanmax((np.abs(got_out - want) / tol)[finite & (tol > 0)])
    live = np.isfinite(wlse)
    assert np.array_equal(got_lse[~live & ~np.isnan(wlse)], wlse[~live & ~np.isnan(wlse)])
    with np.errstate(invalid="ignore"):
        off = np.abs(got_lse - wlse)
    assert (off[live] <= (weight + 4 * E * (1 + np.abs(wlse)))[live]).all()
    return out, lse


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("B,T,H,Hk,D,prefix,lens,ps", [
    (1, 1, 1, 1, 64, 0, [1], 16),                       # one key
    (2, 1, 8, 2, 64, 40, [50, 41], 16),                 # a prefix that ends inside a page
    (3, 1, 4, 4, 128, 64, [64, 65, 200], 16),           # nothing of its own; every head its own keys
    (2, 5, 8, 1, 128, 100, [105, 300], 8),              # drafts
    (4, 3, 10, 2, 80, 33, [36, 90, 35, 33], 24),        # dim and page size that are no powers of two
    (2, 2, 6, 2, 96, 0, [2, 77], 1),                    # pages of one token
    (2, 1, 16, 1, 192, 128, [129, 260], 32),
    (1, 17, 5, 1, 256, 31, [48], 7),                    # more rows than one tile; long heads
    (2, 1, 3, 3, 8, 5, [9, 6], 16),                     # the shortest heads of 16-bit types
    (70, 1, 8, 2, 64, 300, [301 + i for i in range(70)], 16),   # several row blocks of the prefix
    (5, 1, 4, 1, 128, 1500, [1500 + 40 * i + 1 for i in range(5)], 64),
], ids=lambda v: str(len(v)) if isinstance(v, list) else str(v))
def test_shapes(dtype, B, T, H, Hk, D, prefix, lens, ps):
    args = make(B, T, H, Hk, D, prefix, lens, ps, dtype, seed=B * 100 + D)
    check(*args, prefix)


@pytest.mark.parametrize("dtype", TYPES[:2], ids=str)
@pytest.mark.parametrize("B,T,H,Hk,D,prefix,ps", [
    (33, 1, 1, 1, 64, 1, 16), (40, 1, 2, 2, 128, 64, 16), (11, 3, 4, 4, 40, 65, 8), (9, 1, 8, 2, 128, 700, 24), (12, 5, 6, 2, 80, 129, 1), (20, 1, 16, 2, 96, 500, 64), (5, 2, 32, 2, 192, 333, 16),
    (9, 4, 16, 1, 256, 200, 32), (3, 17, 24, 2, 136, 450, 16), (33, 2, 16, 4, 128, 2100, 16),
], ids=str)
def test_many_rows_on_the_prefix(dtype, B, T, H, Hk, D, prefix, ps):
    args = make(B, T, H, Hk, D, prefix, [prefix + T + (7 * i) % 50 for i in range(B)], ps, dtype, seed=D + prefix)
    clean, _ = check(*args, prefix)
    # some sequences end inside the prefix, one before it: their row blocks go another way, and the others' results stay
    lens = args[4].clone()
    lens[B // 2], lens[B - 1] = prefix // 2, 0
    out, _ = check(*args[:4], lens, prefix)
    same = [b for b in range(B) if b not in (B // 2, B - 1)]
    assert (out[same].float() - clean[same].float()).abs().max() <= 4 * HALF[dtype] * clean.float().abs().max()


@pytest.mark.parametrize("dtype", TYPES[:2], ids=str)
@pytest.mark.parametrize("B,H,Hk,D,prefix", [(40, 4, 2, 64, 37), (40, 4, 2, 64, 101), (70, 8, 2, 64, 999), (70, 8, 2, 128, 1333), (40, 2, 1, 128, 205), (9, 32, 4, 200, 150), (300, 4, 4, 128, 66)])
def test_nothing_behind_a_prefix_that_ends_inside_a_page(dtype, B, H, Hk, D, prefix):
    # the first sequence ends with the prefix: behind it, in the same page, its slots hold NaN
    args = make(B, 1, H, Hk, D, prefix, [prefix] + [prefix + 1 + i % 9 for i in range(1, B)], 16, dtype, seed=prefix)
    check(*args, prefix)


@pytest.mark.parametrize("dtype", TYPES[:2], ids=str)
@pytest.mark.parametrize("B,Hk,D,prefix,ps", [(33, 32, 64, 60013, 16), (300, 8, 128, 30001, 32), (40, 64, 64, 45000, 64)])
def test_long_prefixes_of_many_rows(dtype, B, Hk, D, prefix, ps):
    # ranges of more tiles than addresses are kept for: against products in 64 bits on the GPU
    g = torch.Generator(device="cuda").manual_seed(prefix)
    shared, M = prefix // ps, prefix // ps + 2
    P = shared + 2 * B
    table = torch.empty((B, M), dtype=torch.int64, device="cuda")
    ids = torch.randperm(P, generator=g, device="cuda")
    table[:, :shared], table[:, shared:] = ids[:shared], ids[shared:].reshape(B, 2)
    k, v = (torch.randn((P, ps, Hk, D), generator=g, device="cuda").to(dtype) for _ in range(2))
    left = prefix - shared * ps
    for x in (k, v):
        x[table[1:, shared], :left] = x[table[0, shared], :left].clone()
    q = torch.randn((B, 1, Hk, D), generator=g, device="cuda").to(dtype)
    lens = torch.full((B,), prefix, dtype=torch.int32, device="cuda")
    out, lse = atk.shared_prefix_attention(q, k, v, table.int(), lens, prefix, return_lse=True)
    h = HALF[dtype]
    for head in range(Hk):
        kk, vv = (x[table[0], :, head].reshape(-1, D)[:prefix].double() for x in (k, v))
        s = q[:, 0, head].double() @ kk.t() * D ** -0.5
        w = torch.softmax(s, 1)
        want, mass = w @ vv, w @ vv.abs()
        weight = 2 * (D + 4) * E * D ** -0.5 * (q[:, 0, head].double().abs() @ kk.abs().t()).amax(1) + (4 + prefix) * E
        tol = mass * (h + 2 * weight)[:, None] + h * want.abs()
        if dtype == torch.float16:
            tol = tol + 2 * prefix * vv.abs().max() * 2.0 ** -31 + 2.0 ** -24
        assert ((out[:, 0, head].double() - want).abs() <= tol).all()
        wlse = torch.logsumexp(s, 1)
        assert ((lse[:, 0, head].double() - wlse).abs() <= weight + 4 * E * (1 + wlse.abs())).all()


@pytest.mark.parametrize("dtype", TYPES[:2], ids=str)
def test_many_rows_with_scores_at_the_ends(dtype):
    q, k, v, table, lens = make(40, 1, 4, 2, 64, 300, [301] * 40, 16, dtype, seed=8, scale_q=20.0)
    check(q, k, v, table, lens, 300, scale=1.0)
    check(q, k, v, table, lens, 300, scale=1e-6)
    q = q.abs()
    one = k.clone()
    one[table[0, 3].long(), 3] = float("-inf")
    check(q, one, v, table, lens, 300)
    k = torch.where(torch.isnan(k), k, torch.full_like(k, float("-inf")))
    out, lse = check(q, k, v, table, lens, 300)
    assert (out == 0).all() and (lse == float("-inf")).all()
    one = k.clone()
    one[table[0, 3].long(), 3] = float("nan")     # a key that all see
    out, lse = check(q, one, v, table, lens, 300)
    assert torch.isnan(out[:, :, 0]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_rows_that_see_nothing(dtype):
    # empty sequences, sequences shorter than their new tokens, and ones that end inside the prefix
    q, k, v, table, lens = make(6, 4, 4, 2, 64, 40, [60, 44, 41, 44, 44, 44], 16, dtype, seed=3)
    lens = torch.tensor([60, 0, 2, 1, 40, 21], dtype=torch.int32, device="cuda")
    out, lse = check(q, k, v, table, lens, 40)
    assert (out[1] == 0).all() and (lse[1] == float("-inf")).all() and (out[2, :2] == 0).all() and not (out[2, 2:] == 0).all()
    check(q, k, v, table, lens, 0)
    lens = torch.zeros((6,), dtype=torch.int32, device="cuda")
    out, lse = check(q, k, v, table, lens, 0)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("wide", [False, True])
def test_masked_values_have_no_influence(dtype, value, wide):
    # the last new token's key and value are not finite: the queries before it do not see them
    q, k, v, table, lens = make(3, 4, 8, 2, 64, 33, [37, 70, 50], 16, dtype, seed=9)
    if wide:
        table = wider(table, 16)
    clean, _ = _check(q, k, v, table, lens, 33, None, None)
    for b in range(3):
        n = int(lens[b]) - 1
        k[table[b, n // 16].long(), n % 16] = value
        v[table[b, n // 16].long(), n % 16] = value
    out, lse = atk.shared_prefix_attention(q, k, v, table, lens, 33, return_lse=True)
    assert torch.equal(out[:, :3], clean[:, :3]) and not torch.isfinite(out[:, 3]).all()
    # within the prefix, for a sequence that ends there
    lens[1] = 20
    clean, _ = atk.shared_prefix_attention(q, k, v, table, lens, 33, return_lse=True)
    v[table[0, 1].long(), 16 - 16 + 8] = value  # key 24
    out, _ = atk.shared_prefix_attention(q, k, v, table, lens, 33, return_lse=True)
    assert torch.equal(out[1], clean[1]) and not torch.isfinite(out[0, 0]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_scores_at_the_ends_of_the_range(dtype):
    q, k, v, table, lens = make(2, 2, 4, 2, 64, 30, [40, 33], 16, dtype, seed=5, scale_q=20.0)
    check(q, k, v, table, lens, 30, scale=1.0)          # one key takes it all
    check(q, k, v, table, lens, 30, scale=1e-6)         # all alike
    # keys of -inf: weight 0 beside others; a row of nothing else is empty
    q = q.abs()
    one = k.clone()
    one[table[0, 0].long(), 3] = float("-inf")
    check(q, one, v, table, lens, 30)
    k = torch.where(torch.isnan(k), k, torch.full_like(k, float("-inf")))
    out, lse = check(q, k, v, table, lens, 30)
    assert (out == 0).all() and (lse == float("-inf")).all()


def test_lowest_finite_scores():
    # scores near the lowest finite number: still a softmax over them
    q, k, v, table, lens = make(1, 1, 2, 1, 64, 0, [20], 16, torch.float32, seed=6)
    k = torch.where(torch.isnan(k), k, torch.full_like(k, -3.0e38))
    q = torch.zeros_like(q)
    q[..., 0] = 1.0
    out, _ = atk.shared_prefix_attention(q, k, v, table, lens, 0, scale=1.0, return_lse=True)
    want = torch.stack([v[table[0, j // 16].long(), j % 16, 0] for j in range(20)]).double().mean(0)
    assert torch.isfinite(out).all() and (out[0, 0, 0].double() - want).abs().max() <= 64 * E * 4


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_strides_rows_and_out(dtype):
    B, T, H, Hk, D = 3, 2, 8, 4, 64
    q, k, v, table, lens = make(B, T, H, Hk, D, 40, [50, 60, 45, 48, 70], 16, dtype, seed=11, head_major=True, rows=5)
    seqs = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    table[4, :2] = table[0, :2]
    k[table[4, 2].long(), :8] = k[table[0, 2].long(), :8]
    v[table[4, 2].long(), :8] = v[table[0, 2].long(), :8]
    wide = torch.full((B, T, H + 2 * Hk, D), 7.0, dtype=dtype, device="cuda")   # q as a part of a fused projection
    wide[:, :, :H] = q
    long_table = torch.full((5, table.shape[1] + 3), -1, dtype=torch.int32, device="cuda")
    long_table[:, :table.shape[1]] = table
    plain = check(q, k, v, table, lens, 40, seqs=seqs)
    out = torch.zeros((T, B, H, D), dtype=dtype, device="cuda").transpose(0, 1)
    got, lse = atk.shared_prefix_attention(wide[:, :, :H], k, v, long_table[:, :table.shape[1]], lens, 40, seqs=seqs, out=out, return_lse=True)
    assert got is out and torch.equal(out, plain[0]) and torch.equal(lse, plain[1])
    only = atk.shared_prefix_attention(q, k.contiguous(), v.contiguous(), table, lens, 40, seqs=seqs)
    assert torch.equal(only, plain[0])


def test_same_result_every_time_and_on_other_streams():
    args = make(20, 1, 8, 2, 128, 900, [901 + 7 * i for i in range(20)], 16, torch.bfloat16, seed=12)
    want = atk.shared_prefix_attention(*args, 900, return_lse=True)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(atk.shared_prefix_attention(*args, 900, return_lse=True))
    torch.cuda.synchronize()
    for g in got:
        assert torch.equal(g[0], want[0]) and torch.equal(g[1], want[1])


@pytest.mark.parametrize("keys", [0, 2048])
def test_graph_follows_lengths(keys):
    q, k, v, table, lens = make(4, 1, 8, 2, 64, 100, [164, 150, 130, 120], 16, torch.float16, seed=13)
    table = wider(table, 16, keys)
    out = torch.empty_like(q)
    atk.shared_prefix_attention(q, k, v, table, lens, 100, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        atk.shared_prefix_attention(q, k, v, table, lens, 100, out=out)
    for step in range(4):
        lens.sub_(5)
        q.mul_(1.25)
        want = atk.shared_prefix_attention(q, k, v, table, lens, 100)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), step


@pytest.mark.parametrize("keys", [0, 2048])
def test_bad_numbers_on_the_device(keys):
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    args = make(3, 1, 4, 2, 64, 20, [30, 40, 50], 16, torch.bfloat16, seed=14)
    args[3] = wider(args[3], 16, keys)
    good = atk.shared_prefix_attention(*args, 20, status=status)
    assert status.item() == 0
    q, k, v, table, lens = args
    bad = table.clone()
    bad[1, 2] = 1 << 30
    bad[2, 2] = -5
    out = atk.shared_prefix_attention(q, k, v, bad, lens, 20, status=status)
    assert status.item() == atk.ATK_STATUS_BAD_PAGE and torch.equal(out[0], good[0])
    status.zero_()
    out = atk.shared_prefix_attention(q, k, v, table, lens, 20, seqs=torch.tensor([0, 7, -1], dtype=torch.int32, device="cuda"), status=status)
    assert status.item() == atk.ATK_STATUS_BAD_SEQ and torch.equal(out[0], good[0]) and (out[1:] == 0).all()
    status.zero_()
    out = atk.shared_prefix_attention(q, k, v, table, torch.tensor([30, 1 << 30, -3], dtype=torch.int32, device="cuda"), 20, status=status)
    assert status.item() & atk.ATK_STATUS_BAD_LEN and torch.equal(out[0], good[0]) and (out[2] == 0).all()
    out = atk.shared_prefix_attention(q, k, v, bad, lens, 20)    # without a status: as quiet
    assert torch.equal(out[0], good[0])


def test_shared_keys_are_read_through_the_first_row():
    # the other rows hold nothing there, and the first one is no row: nobody has shared keys then
    for keys in (0, 2048):
        q, k, v, table, lens = make(3, 1, 4, 2, 64, 40, [50, 60, 45], 16, torch.bfloat16, seed=15)
        table = wider(table, 16, keys)
        want = atk.shared_prefix_attention(q, k, v, table, lens, 32)
        table[1:, :2] = -1
        status = torch.zeros((1,), dtype=torch.int32, device="cuda")
        assert torch.equal(atk.shared_prefix_attention(q, k, v, table, lens, 32, status=status), want) and status.item() == 0
        out = atk.shared_prefix_attention(q, k, v, table, lens, 32, seqs=torch.tensor([99, 1, 2], dtype=torch.int32, device="cuda"), status=status)
        assert status.item() == atk.ATK_STATUS_BAD_SEQ and (out[0] == 0).all() and torch.isfinite(out).all()


def test_pages_past_32_bits():
    # pages 2^32 bytes and more apart
    big = torch.empty(((1 << 31) + (1 << 20),), dtype=torch.bfloat16, device="cuda")
    pages = torch.as_strided(big, (2, 16, 2, 64), (1 << 31, 128, 64, 1))
    k = torch.randn((2, 16, 2, 64), device="cuda").bfloat16()
    pages.copy_(k)
    q = torch.randn((1, 1, 4, 64), device="cuda").bfloat16()
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([30], dtype=torch.int32, device="cuda")
    for prefix in (0, 20):
        assert torch.equal(atk.shared_prefix_attention(q, pages, pages, table, lens, prefix), atk.shared_prefix_attention(q, k, k, table, lens, prefix))


def test_nothing_to_do_and_refusals():
    q, k, v, table, lens = make(2, 1, 4, 2, 64, 20, [30, 40], 16, torch.bfloat16)
    assert atk.shared_prefix_attention(q[:, :0], k, v, table, lens, 20).shape == (2, 0, 4, 64)
    with pytest.raises(ValueError, match="prefix_len"):
        atk.shared_prefix_attention(q, k, v, table, lens, 10000)
    with pytest.raises(ValueError, match="contiguous"):
        atk.shared_prefix_attention(q.transpose(2, 3).contiguous().transpose(2, 3), k, v, table, lens, 20)
    with pytest.raises(ValueError, match="divisor"):
        atk.shared_prefix_attention(q[:, :, :3], k, v, table, lens, 20)
    with pytest.raises(TypeError, match="int32"):
        atk.shared_prefix_attention(q, k, v, table, lens.long(), 20)
    with pytest.raises(ValueError, match="fewer rows"):
        atk.shared_prefix_attention(q, k, v, table[:1], lens[:1], 20)
    with pytest.raises(ValueError, match="out must"):
        atk.shared_prefix_attention(q, k, v, table, lens, 20, out=q.float())
    with pytest.raises(atk.ApproxTopkError):
        atk.shared_prefix_attention(q, k, v, table, lens, 20, scale=-1.0)
    with pytest.raises(atk.ApproxTopkError):
        atk.shared_prefix_attention(q[..., :60], k[..., :60], v[..., :60], table, lens, 20)
