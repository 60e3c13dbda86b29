"""quantized_attention where its launch plan changes: 17 to 96 queries and many of them, in one piece and cut into ranges, more row blocks than one, more sequences than are cut; bad pages in each way of
sharing the work.

The definition in 64 bits, a sequence and a head at a time.  The tolerance is that of the other tests of quantized_attention: with h half a step of the type and e = 2^-24, a weight is rounded to the type (h,
against the sum of weight * |v|), so is the result (h of it); a score is a sum of dim products in f32 (f32: of three for each), off by (3 dim + 4) e of scale * sum |q k|, and a weight by as much relatively, in
the sum of weights too; 2^x is good to 4 e; sums over n keys add n e (f32: 3 n).  f16 weights have steps of 2^-31 of the largest at the least."""
import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk
from oracle import quant as oracle

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.bfloat16, torch.float16, torch.float32]
E = 2.0 ** -24


def make(B, T, H, Hk, D, lens, ps, dtype, bits, seed=0):
    """q, k, v, table, lens; unused pages, unused slots and padding hold bytes of NaN, and entries past a row's pages are -1."""
    g = np.random.default_rng(seed)
    rows = len(lens)
    M = max(1, max(-(-n // ps) for n in lens)) + 2
    P = rows * M + 1
    table = g.permutation(P)[:rows * M].reshape(rows, M)
    pools = []
    for _ in range(2):
        pool = np.full((P, ps, oracle.token_bytes(Hk, D, bits)), 0xFF, np.uint8)
        for r in range(rows):
            at = np.arange(lens[r])
            if lens[r]:
                pool[table[r, at // ps], at % ps] = oracle.encode(g.standard_normal((lens[r], Hk, D)), bits)
        pools.append(torch.from_numpy(pool).cuda())
    for r in range(rows):
        table[r, -(-lens[r] // ps):] = -1
    q = torch.from_numpy(g.standard_normal((B, T, H, D))).to(dtype).cuda()
    return [q, *pools, torch.from_numpy(table).int().cuda(), torch.tensor(lens, dtype=torch.int32).cuda()]


def wider(table, ps, keys):
    """The table with room for more pages: the host plans for longer sequences."""
    wide = torch.full((table.shape[0], table.shape[1] + keys // ps), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    return wide


def definition(q, k, v, table, lens, Hk, bits):
    """out, lse and the tolerances of both; keys of pages that are none are not there."""
    B, T, H, D = q.shape
    G, ps, dtype = H // Hk, k.shape[1], q.dtype
    kv = [torch.from_numpy(oracle.decode(p.cpu().numpy(), Hk, D, bits)).to(dtype).double() for p in (k, v)]
    q, table = q.double().cpu(), table.cpu()
    out, lse = torch.zeros((B, T, H, D), dtype=torch.float64), torch.full((B, T, H), -float("inf"), dtype=torch.float64)
    tol, ltol = torch.zeros((B, T, H, D), dtype=torch.float64), torch.zeros((B, T, H), dtype=torch.float64)
    scale, h, f32 = D ** -0.5, HALF[dtype], 3 if dtype == torch.float32 else 1
    for b in range(B):
        n = int(lens[b])
        at = torch.arange(n)
        page = table[b][at // ps].long()
        real = (page >= 0) & (page < k.shape[0])
        kk, vv = (torch.where(real[:, None, None], x[page.clamp(0, k.shape[0] - 1), at % ps], 0.0) for x in kv)
        seen = (at[None, :] < n - (T - 1) + torch.arange(T)[:, None]) & real[None, :]              # (T, n)
        seen = seen[:, None, :].expand(T, G, n).reshape(T * G, n)
        some = seen.any(1)
        for j in range(Hk):
            x = q[b, :, j * G:(j + 1) * G].reshape(T * G, D)
            s = torch.where(seen, scale * (x @ kk[:, j].t()), -float("inf"))
            m = torch.where(some, s.amax(1) if n else torch.zeros(T * G, dtype=torch.float64), 0.0)
            w = torch.exp(s - m[:, None])
            total = torch.where(some, w.sum(1), 1.0)
            w = w / total[:, None]
            size = torch.where(seen, scale * (x.abs() @ kk[:, j].abs().t()), 0.0).amax(1) if n else torch.zeros(T * G, dtype=torch.float64)
            count = seen.sum(1)
            top = torch.where(seen, vv[:, j].abs().amax(1)[None, :], 0.0).amax(1) if n else torch.zeros(T * G, dtype=torch.float64)
            weight = 2 * (f32 * D + 4) * E * size + (4 + f32 * count) * E
            o = w @ vv[:, j]
            t = (w @ vv[:, j].abs()) * (h + 2 * weight)[:, None] + h * o.abs()
            if dtype == torch.float16:
                t = t + 2 * (count * top * 2.0 ** -31)[:, None] + 2.0 ** -24     # (and outputs have subnormal steps)
            l = torch.where(some, m + torch.log(total), -float("inf"))
            lt = weight + 4 * E * (1 + torch.where(some, l, 0.0).abs())
            part = slice(j * G, (j + 1) * G)
            out[b, :, part], lse[b, :, part] = o.reshape(T, G, D), l.reshape(T, G)
            tol[b, :, part], ltol[b, :, part] = t.reshape(T, G, D), lt.reshape(T, G)
    return out, lse, tol, ltol


def check(args, Hk, bits, widths=(0, 3000, 40000), told=0):
    q, k, v, table, lens = args
    want, wlse, tol, ltol = definition(q, k, v, table, lens, Hk, bits)
    live = torch.isfinite(wlse)
    for keys in widths:
        status = torch.zeros((1,), dtype=torch.int32, device="cuda")
        out, lse = atk.quantized_attention(q, k, v, wider(table, k.shape[1], keys), lens, Hk, bits=bits, return_lse=True, status=status)
        out, lse = out.double().cpu(), lse.double().cpu()
        assert status.item() == told, keys
        off = (out - want).abs()
        assert (off <= tol).all(), (keys, (off / tol)[tol > 0].max())
        assert torch.equal(lse[~live], wlse[~live]) and ((lse - wlse).abs()[live] <= ltol[live]).all(), keys


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("B,T,H,Hk,D,lens,ps", [
    (2, 5, 8, 1, 64, [1500, 333], 16),          # 40 queries
    (1, 9, 6, 1, 32, [700], 24),                # 54, of heads with padding
    (2, 5, 8, 2, 128, [1040, 130], 16),         # 20
    (3, 3, 10, 1, 96, [901, 0, 2], 8),          # 30, of heads with padding; queries that see no key
    (2, 2, 36, 4, 64, [1030, 64], 16),          # 18, for a team of heads
    (1, 8, 12, 1, 128, [2100], 16),             # 96, the most that do not share operands
    (1, 97, 1, 1, 64, [1700], 16),              # 97, the least that do
    (1, 33, 3, 1, 96, [1200], 7),               # 99, of heads with padding, pages that are no fours
    (2, 70, 8, 1, 128, [1600, 520], 16),        # 560: row blocks, cut
    (1, 150, 8, 2, 64, [1333], 32),             # 600
    (2, 17, 1, 1, 160, [400, 1100], 16),        # 17, of long heads
    (1, 20, 10, 1, 256, [900], 16),             # 200, of long heads
    (1, 300, 2, 1, 32, [260], 16),              # more new tokens than keys
    (3, 2, 20, 2, 64, [300, 0, 450], 16),       # 20, short rows of the table: several tiles at once, nothing cut
    (2, 5, 5, 1, 128, [390, 31], 16),
    (2, 4, 5, 1, 32, [700, 45], 16),            # 20, of heads with padding
    (2, 8, 5, 1, 96, [500, 1], 16),             # 40, of heads with padding
    (2, 1, 4, 2, 256, [900, 40], 16),           # few, of long heads
], ids=str)
def test_queries(bits, dtype, B, T, H, Hk, D, lens, ps):
    check(make(B, T, H, Hk, D, lens, ps, dtype, bits, seed=T * H + D), Hk, bits)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
@pytest.mark.parametrize("T,Hk,D", [(1, 2, 64), (1, 1, 256), (6, 1, 128), (10, 2, 64), (10, 1, 128), (35, 2, 128), (35, 1, 64), (70, 1, 96)], ids=str)
def test_pages_that_are_none(bits, dtype, T, Hk, D):
    """Entries outside the pool in front of, between and behind good ones, also all that some queries see."""
    ps = 16
    for seed, bad in enumerate(({0: {0: -1, 17: 1 << 30}, 1: {3: -7}}, {0: {j: -1 for j in range(5, 30)}, 1: {21: -(1 << 31)}}, {1: {j: (1 << 31) - 1 for j in range(21)}})):
        args = make(2, T, 4 * Hk, Hk, D, [600, 340], ps, dtype, bits, seed=seed)
        for row, entries in bad.items():
            for j, page in entries.items():
                args[3][row, j] = page
        check(args, Hk, bits, told=atk.ATK_STATUS_BAD_PAGE)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("B,T,H,Hk,D", [(8200, 1, 4, 2, 64), (8200, 4, 5, 1, 64), (8200, 1, 3, 1, 128), (8200, 5, 4, 1, 128), (8200, 2, 3, 1, 96), (8200, 6, 3, 1, 96), (8200, 1, 6, 3, 32),
                                        (8200, 3, 6, 1, 32), (8200, 1, 2, 1, 32), (8200, 9, 12, 1, 32), (9000, 1, 5, 5, 64), (9000, 3, 24, 4, 128), (3000, 1, 8, 1, 64), (3000, 3, 16, 2, 64), (8000, 1, 2, 1, 128)], ids=str)
def test_more_sequences_than_are_cut(bits, dtype, B, T, H, Hk, D):
    """Some thousand sequences, of rows that many of them share: each gets what its row's first one gets, bit for bit."""
    lens = [1, 33, 1030, 0, 200, 7, 64, 65, 300, 129]
    rows = len(lens)
    q, k, v, table, n = make(rows, T, H, Hk, D, lens, 16, dtype, bits, seed=T)
    table = wider(table, 16, 3000)
    seqs = (torch.arange(B, device="cuda") % rows).int()
    out, lse = atk.quantized_attention(q[seqs.long()], k, v, table, n, Hk, bits=bits, seqs=seqs, return_lse=True)
    assert torch.equal(out.reshape(-1, rows, T, H, D), out[:rows].expand(B // rows, rows, T, H, D)) and torch.equal(lse.reshape(-1, rows, T, H), lse[:rows].expand(B // rows, rows, T, H))
    want, wlse, tol, ltol = definition(q, k, v, table, n, Hk, bits)
    live = torch.isfinite(wlse)
    assert ((out[:rows].double().cpu() - want).abs() <= tol).all()
    assert torch.equal(lse[:rows].double().cpu()[~live], wlse[~live]) and ((lse[:rows].double().cpu() - wlse).abs()[live] <= ltol[live]).all()


@pytest.mark.parametrize("T,H,Hk,D", [(70, 8, 2, 128), (5, 8, 1, 64), (5, 8, 2, 128)], ids=str)
def test_captured_and_replayed(T, H, Hk, D):
    """Many queries in a graph, replayed with other inputs and lengths beside the same call outside of it."""
    q, k, v, table, lens = make(2, T, H, Hk, D, [1300, 700], 16, torch.bfloat16, 4, seed=1)
    table = wider(table, 16, 3000)
    x, n = q.clone(), lens.clone()
    atk.quantized_attention(x, k, v, table, n, Hk)     # (what loads on a first call is loaded)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = atk.quantized_attention(x, k, v, table, n, Hk, return_lse=True)
    for step in range(4):
        x.copy_(q.flip(0) if step % 2 else q)
        n.copy_(lens - 37 * step)
        graph.replay()
        want, wlse = atk.quantized_attention(x, k, v, table, n, Hk, return_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wlse)
