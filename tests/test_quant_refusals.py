"""The quantised cache's host side: symbols, sizes, and refusals that come before any HIP call; the oracle's format against float8 of torch."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2412_04358_amd as atk
from oracle import quant as oracle
from paper_2412_04358_amd import decode, quantized

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULLP, UNSUP, DTYPE, ALIGN, WORK, ARGS = -1, -4, -5, -7, -8, -9
FAKE = 1 << 20  # never followed: the checks come first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(atk.lib_path()):
        import __graft_entry__

        __graft_entry__.build()
    return quantized._library()


def test_header_and_library_agree(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "atk_quant.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(atk_[a-z_]+)\s*\(", text))
    assert len(names) == 5
    for n in names:
        assert getattr(lib, n).argtypes is not None, n


@pytest.mark.parametrize("heads,dim,bits", [(1, 32, 4), (8, 128, 4), (8, 128, 8), (5, 96, 4), (3, 256, 8), (2, 64, 4), (7, 160, 8)])
def test_token_bytes(lib, heads, dim, bits):
    assert atk.quantized_token_bytes(heads, dim, bits) == oracle.token_bytes(heads, dim, bits)
    assert oracle.token_bytes(heads, dim, bits) % 16 == 0


@pytest.mark.parametrize("heads,dim,bits,code", [(0, 64, 4, ARGS), (1, 0, 4, ARGS), (1, 48, 4, ARGS), (1, 288, 4, ARGS), (1, -32, 4, ARGS), (1, 64, 2, UNSUP), (1, 64, 16, UNSUP), (1 << 20, 64, 4, ARGS)])
def test_token_bytes_refuses(lib, heads, dim, bits, code):
    assert lib.atk_quant_token_bytes(heads, dim, bits) == code
    with pytest.raises(atk.ApproxTopkError):
        atk.quantized_token_bytes(heads, dim, bits)


def _attention(**kw):
    i3 = ctypes.c_int64 * 3
    a = dict(q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=None, page_table=FAKE, lens=FAKE, seqs=None, status=None, batch=4, tokens=1, heads=8, kv_heads=2, dim=64, page_size=16, n_pages=100,
             rows=4, row_pages=20, table_stride=20, q_stride=(512, 512, 64), out_stride=(512, 512, 64), scale=0.125, dtype=1, bits=4)
    a.update(kw)
    for n in ("q_stride", "out_stride"):
        a[n] = i3(*a[n])
    return quantized._QuantAttentionArgs(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), ARGS), (dict(tokens=0), ARGS), (dict(heads=0), ARGS), (dict(kv_heads=3), ARGS), (dict(kv_heads=0), ARGS), (dict(page_size=0), ARGS), (dict(n_pages=0), ARGS),
    (dict(rows=3), ARGS), (dict(row_pages=0), ARGS), (dict(table_stride=19), ARGS), (dict(scale=0.0), ARGS), (dict(scale=1e-39), ARGS), (dict(scale=1e31), ARGS),
    (dict(scale=-1.0), ARGS), (dict(scale=float("nan")), ARGS), (dict(scale=float("inf")), ARGS), (dict(row_pages=1 << 28, table_stride=1 << 28), ARGS), (dict(batch=1 << 31, seqs=FAKE), ARGS),
    (dict(dim=48), ARGS), (dict(dim=288), ARGS), (dict(dim=0), ARGS), (dict(bits=5), UNSUP), (dict(dtype=3), DTYPE), (dict(dtype=-1), DTYPE),
    (dict(n_pages=1 << 26), ARGS), (dict(page_size=1 << 25, row_pages=1), ARGS),     # pools of 2^36 bytes
    (dict(q_stride=(513, 512, 64)), ALIGN), (dict(out_stride=(512, 512, 60)), ALIGN), (dict(out_stride=(-512, 512, 64)), ARGS), (dict(tokens=1 << 27), ARGS),
])
def test_attention_refuses(lib, kw, code):
    assert lib.atk_quant_attention_workspace_bytes(_attention(**kw)) == code
    assert lib.atk_quant_attention(_attention(**kw), FAKE, 1 << 40, None) == code


@pytest.mark.parametrize("kw,code", [(dict(q=None), NULLP), (dict(k=None), NULLP), (dict(v=None), NULLP), (dict(out=None), NULLP), (dict(page_table=None), NULLP), (dict(lens=None), NULLP),
                                     (dict(q=FAKE + 8), ALIGN), (dict(k=FAKE + 4), ALIGN), (dict(v=FAKE + 8), ALIGN), (dict(lens=FAKE + 2), ALIGN), (dict(lse=FAKE + 1), ALIGN),
                                     (dict(status=FAKE + 2), ALIGN)])
def test_attention_refuses_pointers(lib, kw, code):
    assert lib.atk_quant_attention(_attention(**kw), FAKE, 1 << 40, None) == code


@pytest.mark.parametrize("kw", [dict(), dict(row_pages=2000, table_stride=2000), dict(tokens=50), dict(dtype=0, tokens=9), dict(dim=256, bits=8, q_stride=(2048, 2048, 256), out_stride=(2048, 2048, 256))])
def test_attention_workspace(lib, kw):
    need = lib.atk_quant_attention_workspace_bytes(_attention(**kw))
    assert need > 0
    assert lib.atk_quant_attention(_attention(**kw), FAKE, need - 1, None) == WORK
    assert lib.atk_quant_attention(_attention(**kw), FAKE + 4, need, None) == ALIGN
    assert lib.atk_quant_attention(_attention(**kw), None, need, None) == NULLP


def _tables(**kw):
    a = dict(page_table=FAKE, lens=FAKE, refs=FAKE, free_pages=FAKE, n_free=FAKE, status=FAKE, work=FAKE, rows=4, row_pages=8, n_pages=64, page_size=16, work_bytes=1 << 20)
    a.update(kw)
    return decode._Tables(**a)


def test_pages_refuse(lib):
    one, none = (ctypes.c_void_p * 1)(FAKE), (ctypes.c_void_p * 1)(None)
    strides = (ctypes.c_int64 * 2)(4096, 256)

    def both(code, table=_tables(), pools=one, others=one, strides=strides, n_pools=1, heads=2, dim=64, bits=4, dtype=1, seqs=FAKE, n=2, tokens=3):
        assert lib.atk_append_quantized(table, pools, others, strides, n_pools, heads, dim, bits, dtype, seqs, n, tokens, None) == code
        assert lib.atk_read_quantized(table, pools, others, n_pools, heads, dim, bits, dtype, seqs, None, n, tokens, None) == code

    for kw, code in [(dict(rows=0), ARGS), (dict(row_pages=0), ARGS), (dict(n_pages=0), ARGS), (dict(page_size=0), ARGS), (dict(row_pages=1 << 27), ARGS), (dict(lens=None), NULLP),
                     (dict(work=None), NULLP), (dict(refs=FAKE + 2), ALIGN), (dict(work=FAKE + 8), ALIGN), (dict(work_bytes=100), WORK)]:
        both(code, table=_tables(**kw))
    both(NULLP, pools=none)
    both(NULLP, others=none)
    both(NULLP, seqs=None)
    both(ALIGN, seqs=FAKE + 2)
    both(ALIGN, pools=(ctypes.c_void_p * 1)(FAKE + 8))
    both(ALIGN, others=(ctypes.c_void_p * 1)(FAKE + 8))
    both(DTYPE, dtype=3)
    both(UNSUP, bits=3)
    both(ARGS, dim=40)
    both(ARGS, heads=0)
    both(ARGS, n=-1)
    both(ARGS, tokens=-1)
    both(ARGS, n_pools=-1)
    both(0, n=0)
    both(0, tokens=0)
    t = _tables()
    assert lib.atk_append_quantized(t, one, one, strides, 1, 2, 64, 4, 1, FAKE, 5, 1, None) == ARGS        # more sequences than rows
    assert lib.atk_append_quantized(t, one, one, None, 1, 2, 64, 4, 1, FAKE, 2, 1, None) == NULLP
    assert lib.atk_append_quantized(t, one, one, (ctypes.c_int64 * 2)(-16, 256), 1, 2, 64, 4, 1, FAKE, 2, 1, None) == ARGS
    assert lib.atk_append_quantized(t, one, one, (ctypes.c_int64 * 2)(4096, 264), 1, 2, 64, 4, 1, FAKE, 2, 2, None) == ALIGN
    assert lib.atk_read_quantized(t, one, one, 1, 2, 64, 4, 1, FAKE, FAKE + 1, 2, 1, None) == ALIGN
    assert lib.atk_read_quantized(t, one, one, 1, 2, 64, 4, 1, FAKE, None, 1 << 30, 1 << 30, None) == ARGS


def test_python_refuses_tensors_elsewhere(lib):
    q = torch.zeros((2, 1, 4, 64))
    pool = torch.zeros((4, 16, atk.quantized_token_bytes(2, 64)), dtype=torch.uint8)
    table, lens = torch.zeros((2, 4), dtype=torch.int32), torch.ones((2,), dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        atk.quantized_attention(q, pool, pool, table, lens, 2)
    with pytest.raises(ValueError, match="must be"):
        atk.quantized_attention(q[0], pool, pool, table, lens, 2)
    with pytest.raises(TypeError, match="float32"):
        atk.quantized_attention(q.double(), pool, pool, table, lens, 2)


def test_the_oracles_ladder_is_float8():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, oracle.ladder(8))
    # whole codes: what torch rounds to, where the block's unit is 1 (largest magnitude 256 to 448)
    x = torch.linspace(-448, 448, 32 * 500, dtype=torch.float32).reshape(500, 1, 32).clone()
    x[:, :, 0] = 300.0
    got = oracle.decode(oracle.encode(x.numpy(), 8), 1, 32, 8)
    assert np.array_equal(got, x.to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("bits", [4, 8])
def test_the_oracles_nearest(bits):
    x = np.random.default_rng(0).standard_normal((200, 3, 64))
    got = oracle.decode(oracle.encode(x, bits), 3, 64, bits)
    unit = 2.0 ** (np.floor(np.log2(np.abs(x.reshape(200, -1, 32)).max(-1))) - (2 if bits == 4 else 8))
    grid = np.concatenate([oracle.ladder(bits), -oracle.ladder(bits)])
    all_of = (grid * unit[..., None, None]).reshape(200, 6, 1, -1)
    best = np.abs(all_of - x.reshape(200, 6, 32, 1)).min(-1)
    assert np.array_equal(np.abs(got.reshape(200, 6, 32) - x.reshape(200, 6, 32)), best)
