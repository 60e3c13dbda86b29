"""append_quantized and read_quantized against the formats' ladders, bit for bit: types, heads, odd lengths, shared pages, strides, many pools, what is refused on the device."""
import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk
from oracle import quant as oracle

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def pools_of(n, pages, ps, heads, dim, bits, fill=0xA5):
    return [torch.full((pages, ps, atk.quantized_token_bytes(heads, dim, bits)), fill, dtype=torch.uint8, device="cuda") for _ in range(n)]


def some(shape, dtype, seed):
    """Values over many orders of magnitude, with zeros, middles between codes, and blocks of one value."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(2 * torch.randn((*shape[:-1], 1), generator=g))
    x = torch.where(torch.rand(shape, generator=g) < 0.2, torch.randint(-24, 25, shape, generator=g).float() / 4, x)
    x[torch.rand(shape[:-1], generator=g) < 0.05] = 0
    return x.to(dtype).cuda()


def rows_of(t, pool, row):
    """Bytes of the tokens that a row holds."""
    n, ps = int(t.lens[row]), t.page_size
    table = t.page_table[row].cpu().numpy()
    p = pool.cpu().numpy()
    return np.stack([p[table[j // ps], j % ps] for j in range(n)]) if n else np.zeros((0, p.shape[2]), np.uint8)


def expect(x, bits):
    x = x.double().cpu().numpy()
    return oracle.encode(x.reshape(-1, *x.shape[-2:]), bits).reshape(*x.shape[:-2], oracle.token_bytes(*x.shape[-2:], bits))


def body(rows, heads, dim, bits):
    return rows[..., :heads * dim * bits // 8 + heads * dim // 32]


def same(got, rows, heads, dim, bits, dtype):
    """What is read against the ladder's values, rounded to the type once."""
    want = torch.from_numpy(oracle.decode(rows, heads, dim, bits)).to(dtype)
    got = got.cpu()
    assert got.dtype is dtype and got.shape == want.shape
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,held,T,heads,dim,ps,n_pools", [
    (1, 0, 1, 1, 32, 16, 1),
    (3, 5, 1, 2, 64, 16, 2),
    (2, 15, 18, 5, 96, 8, 2),        # over page borders, rows with padding
    (4, 1, 7, 3, 128, 1, 1),         # pages of one token
    (1, 3, 700, 8, 128, 24, 2),      # several pieces of one sequence
    (2, 0, 301, 1, 256, 64, 3),
    (5, 2, 2, 7, 160, 16, 70),       # more pools than a launch has
], ids=str)
def test_append_and_read(bits, dtype, n, held, T, heads, dim, ps, n_pools):
    row_pages = -(-(held + T) // ps) + 1
    t = atk.PageTables.empty(n * row_pages + 2, ps, n + 1, row_pages)
    pools = pools_of(n_pools, n * row_pages + 2, ps, heads, dim, bits)
    seqs = torch.randperm(n + 1, generator=torch.Generator().manual_seed(1))[:n].int().cuda()
    a, b = [some((n, held, heads, dim), dtype, p) for p in range(n_pools)], [some((n, T, heads, dim), dtype, 100 + p) for p in range(n_pools)]
    if held:
        atk.append_quantized(t, pools, seqs, a, bits=bits)
    atk.append_quantized(t, pools, seqs, b, bits=bits)
    torch.cuda.synchronize()
    assert t.status.item() == 0 and t.lens[seqs.long()].tolist() == [held + T] * n
    for p in sorted({0, 1, n_pools // 2, n_pools - 1} & set(range(n_pools))):
        want = np.concatenate([expect(a[p], bits), expect(b[p], bits)], 1)
        for i in range(n):
            assert np.array_equal(body(rows_of(t, pools[p], int(seqs[i])), heads, dim, bits), body(want[i], heads, dim, bits)), (p, i)
    # read, in every type, from places of their own, one sequence twice; before the first and behind the last token lies nothing
    rows = torch.cat([seqs, seqs[:1]])
    starts = ints(*[(held + T) // (i + 1) - 2 for i in range(n)], -3)
    for out_type in TYPES:
        got = atk.read_quantized(t, pools, rows, starts, T + 4, heads, dim, bits=bits, dtype=out_type)
        whole = atk.read_quantized(t, pools, rows, None, held + T, heads, dim, bits=bits, dtype=out_type)
        for p in {0, n_pools - 1}:
            want = np.concatenate([expect(a[p], bits), expect(b[p], bits)], 1)
            want = np.concatenate([want, want[:1]], 0)
            same(whole[p], want, heads, dim, bits, out_type)
            part = np.zeros((n + 1, T + 4, want.shape[2]), np.uint8)
            for i in range(n + 1):
                for x in range(T + 4):
                    if 0 <= starts[i] + x < held + T:
                        part[i, x] = want[i, int(starts[i]) + x]
            same(got[p], part, heads, dim, bits, out_type)
    assert t.status.item() == 0


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_extremes(bits, dtype):
    """The type's smallest and largest numbers, infinities and NaN in single blocks, every exponent."""
    info = torch.finfo(dtype)
    x = torch.zeros((1, 40, 1, 64), dtype=dtype)
    g = torch.Generator().manual_seed(3)
    for j in range(40):
        e = info.tiny * 2.0 ** -3 if j == 0 else 2.0 ** (np.log2(info.tiny) + (np.log2(info.max) - np.log2(info.tiny)) * j / 40)
        x[0, j, 0] = ((2 * torch.rand((64,), generator=g, dtype=torch.float64) - 1) * e).to(dtype)
    x[0, 1, 0, :32] = info.tiny
    x[0, 2, 0, 5] = info.max
    x[0, 3, 0, 40] = -info.max
    x[0, 4, 0, 7] = float("nan")
    x[0, 5, 0, 33] = float("inf")
    x[0, 6, 0, 31] = -float("inf")
    x[0, 7, 0, :32] = -0.0
    x[0, 8, 0, :32] = info.max
    x = x.cuda()
    t = atk.PageTables.empty(4, 16, 1, 4)
    pools = pools_of(1, 4, 16, 1, 64, bits)
    atk.append_quantized(t, pools, ints(0), [x], bits=bits)
    want = expect(x, bits)[0]
    assert np.array_equal(body(rows_of(t, pools[0], 0), 1, 64, bits), body(want, 1, 64, bits))
    for out_type in TYPES:
        same(atk.read_quantized(t, pools, ints(0), None, 40, 1, 64, bits=bits, dtype=out_type)[0][0], want, 1, 64, bits, out_type)
    # values that a 16-bit type has come back as numbers of it
    back = atk.read_quantized(t, pools, ints(0), None, 40, 1, 64, bits=bits, dtype=dtype)[0]
    assert torch.isfinite(back[0, 8:]).all() and torch.isfinite(back[0, 2:4]).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_any_bytes_are_read(bits):
    """Every code under every exponent, also those that are never written."""
    heads, dim = 1, 256
    pools = pools_of(1, 256, 1, heads, dim, bits)
    g = torch.Generator().manual_seed(0)
    pools[0].copy_(torch.randint(0, 256, pools[0].shape, generator=g).to(torch.uint8))
    codes = dim * bits // 8
    pools[0][:, 0, codes:codes + 8] = torch.arange(256, dtype=torch.uint8)[:, None].cuda()
    if bits == 8:
        pools[0][:, 0, :codes] = torch.arange(256, dtype=torch.uint8).cuda()
    t = atk.PageTables(torch.arange(256, dtype=torch.int32, device="cuda").reshape(1, 256).contiguous(), ints(256), torch.ones(256, dtype=torch.int32, device="cuda"),
                       torch.zeros(256, dtype=torch.int32, device="cuda"), ints(0), 1)
    rows = pools[0][:, 0].cpu().numpy()
    for out_type in TYPES:
        same(atk.read_quantized(t, pools, ints(0), None, 256, heads, dim, bits=bits, dtype=out_type)[0][0], rows, heads, dim, bits, out_type)


def test_strided_values():
    """Keys and values as slices of one projection, and one sequence's as an expanded view."""
    n, T, heads, dim = 3, 5, 2, 64
    both = some((n, T, 2 * heads, dim), torch.bfloat16, 0)
    k, v = both[:, :, :heads], both[:, :, heads:]
    t = atk.PageTables.empty(6, 16, 4, 2)
    pools = pools_of(3, 6, 16, heads, dim, 4)
    wide = some((1, T, heads, dim), torch.bfloat16, 1).expand(n, T, heads, dim)
    atk.append_quantized(t, pools, ints(2, 0, 1), [k, v, wide])
    for pool, x in zip(pools, (k, v, wide)):
        for i, row in enumerate((2, 0, 1)):
            assert np.array_equal(body(rows_of(t, pool, row), heads, dim, 4), body(expect(x[i], 4), heads, dim, 4))


def test_shared_pages_are_copied_and_pools_move():
    """Samples of a prompt: fork, append to each, compact; then the parent is still what it was."""
    heads, dim, bits = 2, 96, 4
    t = atk.PageTables.empty(40, 8, 6, 6)
    pools = pools_of(2, 40, 8, heads, dim, bits)
    prompt = [some((1, 13, heads, dim), torch.float16, s) for s in (0, 1)]
    atk.append_quantized(t, pools, ints(0), prompt)
    atk.fork_sequences(t, pools, ints(0, 0, 0, 0), ints(1, 2, 3, 4))
    new = [some((5, 4, heads, dim), torch.float16, s) for s in (2, 3)]
    atk.append_quantized(t, pools, ints(4, 0, 1, 2, 3), new)
    atk.free_sequences(t, ints(2))
    atk.compact_pages(t, pools)
    assert t.status.item() == 0
    for p in range(2):
        for i, row in enumerate((4, 0, 1, 2, 3)):
            if row == 2:
                continue
            want = np.concatenate([expect(prompt[p][0], bits), expect(new[p][i], bits)])
            assert np.array_equal(body(rows_of(t, pools[p], row), heads, dim, bits), body(want, heads, dim, bits))
    # rows that hold one part-filled page at the call, without a fork's copy
    t = atk.PageTables(ints(0, -1, 0, -1).reshape(2, 2).contiguous(), ints(3, 3), ints(2, 0, 0, 0), ints(3, 2, 1, 0), ints(3), 8)
    pools = pools_of(1, 4, 8, heads, dim, bits)
    old = pools[0][0].clone()
    x = some((2, 2, heads, dim), torch.float16, 9)
    atk.append_quantized(t, pools, ints(0, 1), [x])
    assert t.status.item() == 0 and torch.equal(pools[0][0], old) and t.page_table[:, 0].tolist() == [1, 2] and t.refs.tolist()[:3] == [0, 1, 1]
    for i in range(2):
        got = rows_of(t, pools[0], i)
        assert np.array_equal(got[:3], old[:3].cpu().numpy())
        assert np.array_equal(body(got[3:], heads, dim, bits), body(expect(x[i], bits), heads, dim, bits))


def test_all_or_nothing_and_reports():
    heads, dim = 1, 64
    for case, status in (("pages", atk.ATK_STATUS_NO_PAGES), ("row", atk.ATK_STATUS_BAD_SEQ), ("long", atk.ATK_STATUS_BAD_LEN)):
        t = atk.PageTables.empty(3, 4, 3, 2)
        pools = pools_of(1, 3, 4, heads, dim, 4)
        before = pools[0].clone()
        T, seqs = {"pages": (5, ints(0, 1)), "row": (1, ints(0, 3)), "long": (9, ints(0, 1))}[case]
        atk.append_quantized(t, pools, seqs, [some((2, T, heads, dim), torch.bfloat16, 0)])
        torch.cuda.synchronize()
        assert t.status.item() == status and torch.equal(pools[0], before) and t.lens.tolist() == [0, 0, 0] and t.n_free.item() == 3
    # reading: a row that is none, a length that is none, a page that is none
    t = atk.PageTables(ints(0, 7, 1, -1, 2, 2).reshape(3, 2).contiguous(), ints(6, -1, 99), ints(1, 1, 1), ints(0, 0, 0), ints(0), 4)
    pools = pools_of(1, 3, 4, heads, dim, 4, fill=0x22)
    for row, bits_of, there in ((0, atk.ATK_STATUS_BAD_PAGE, 4), (1, atk.ATK_STATUS_BAD_LEN, 0), (2, atk.ATK_STATUS_BAD_LEN, 8), (3, atk.ATK_STATUS_BAD_SEQ, 0), (-1, atk.ATK_STATUS_BAD_SEQ, 0)):
        t.status.zero_()
        got = atk.read_quantized(t, pools, ints(row), None, 10, heads, dim)[0]
        assert t.status.item() == bits_of, row
        assert (got[0, :there] != 0).all() and (got[0, there:] == 0).all(), row


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_large_reads(dtype):
    """More than half of what the caches hold: outputs go past them."""
    heads, dim, T = 8, 128, 1100
    t = atk.PageTables.empty(40, 32, 1, 40)
    pools = pools_of(1, 40, 32, heads, dim, 4)
    atk.append_quantized(t, pools, ints(0), [some((1, T, heads, dim), dtype, 0)])
    rows, starts = torch.zeros((70,), dtype=torch.int32, device="cuda"), torch.arange(70, dtype=torch.int32, device="cuda")
    one = atk.read_quantized(t, pools, ints(0), None, T + 70, heads, dim, dtype=dtype)[0][0]
    got = atk.read_quantized(t, pools, rows, starts, T, heads, dim, dtype=dtype)[0]
    for i in (0, 1, 33, 69):
        assert torch.equal(got[i], one[i:i + T])
    assert (got[69, T - 69:] == 0).all() and t.status.item() == 0


def test_nothing_to_do():
    t = atk.PageTables.empty(3, 4, 3, 2)
    pools = pools_of(1, 3, 4, 1, 64, 4)
    none = torch.zeros((0,), dtype=torch.int32, device="cuda")
    atk.append_quantized(t, pools, none, [torch.zeros((0, 3, 1, 64), device="cuda")])
    atk.append_quantized(t, pools, ints(0), [torch.zeros((1, 0, 1, 64), device="cuda")])
    assert atk.read_quantized(t, pools, none, None, 3, 1, 64)[0].shape == (0, 3, 1, 64)
    assert atk.read_quantized(t, pools, ints(0), None, 0, 1, 64)[0].shape == (1, 0, 1, 64)
    assert atk.read_quantized(t, [], ints(0), None, 2, 1, 64) == []
    assert t.status.item() == 0 and t.lens.tolist() == [0, 0, 0]


def test_python_refuses():
    t = atk.PageTables.empty(3, 4, 3, 2)
    pools = pools_of(1, 3, 4, 1, 64, 4)
    x = torch.zeros((1, 2, 1, 64), device="cuda")
    with pytest.raises(ValueError, match="equally many"):
        atk.append_quantized(t, pools, ints(0), [x, x])
    with pytest.raises(ValueError, match="needs a pool"):
        atk.append_quantized(t, [], ints(0), [])
    with pytest.raises(TypeError, match="uint8"):
        atk.append_quantized(t, [pools[0].view(torch.int8)], ints(0), [x])
    with pytest.raises(ValueError, match="shape"):
        atk.append_quantized(t, pools, ints(0), [x], bits=8)
    with pytest.raises(ValueError, match="contiguous"):
        atk.append_quantized(t, pools, ints(0), [torch.zeros((1, 2, 1, 128), device="cuda")[..., ::2]])
    with pytest.raises(ValueError, match="one type"):
        atk.append_quantized(t, pools * 2, ints(0), [x, x.half()])
    with pytest.raises(TypeError, match="float32"):
        atk.append_quantized(t, pools, ints(0), [x.double()])
    with pytest.raises(ValueError, match="GPU"):
        atk.append_quantized(t, pools, ints(0), [x.cpu()])
    with pytest.raises(TypeError, match="dtype"):
        atk.read_quantized(t, pools, ints(0), None, 2, 1, 64, dtype=torch.float64)
    with pytest.raises(TypeError, match="int32"):
        atk.read_quantized(t, pools, ints(0).long(), None, 2, 1, 64)
    with pytest.raises(ValueError, match="starts"):
        atk.read_quantized(t, pools, ints(0), ints(0, 1), 2, 1, 64)
    with pytest.raises(ValueError, match="negative"):
        atk.read_quantized(t, pools, ints(0), None, -1, 1, 64)


def test_captured_and_replayed():
    heads, dim, n = 2, 64, 3
    t = atk.PageTables.empty(64, 4, n, 16)
    pools = pools_of(2, 64, 4, heads, dim, 4)
    seqs = ints(0, 1, 2)
    x = [some((n, 1, heads, dim), torch.bfloat16, s) for s in (0, 1)]
    atk.append_quantized(t, pools, seqs, x)      # (what loads on a first call is loaded)
    atk.read_quantized(t, pools, seqs, None, 12, heads, dim)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        atk.append_quantized(t, pools, seqs, x)
        got = atk.read_quantized(t, pools, seqs, None, 12, heads, dim)
    history = [[y.clone() for y in x]]
    for step in range(6):
        for y, seed in zip(x, (10 + step, 20 + step)):
            y.copy_(some(y.shape, y.dtype, seed))
        history.append([y.clone() for y in x])
        graph.replay()
        torch.cuda.synchronize()
        for p in range(2):
            want = torch.from_numpy(oracle.decode(np.concatenate([expect(h[p], 4) for h in history], 1), heads, dim, 4)).bfloat16()
            assert torch.equal(got[p][:, :step + 2].cpu(), want) and (got[p][:, step + 2:] == 0).all()
    assert t.status.item() == 0
