"""The workspace of quantized_attention against what it returns: sequences that are not cut have as few parts as they can, and calls without parts are not refused for the size of their join."""
import ctypes
import os

import pytest

import paper_2412_04358_amd as atk
from paper_2412_04358_amd import quantized


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(atk.lib_path()):
        import __graft_entry__

        __graft_entry__.build()
    return quantized._library()


def args(batch, tokens, heads, kv_heads, dim, bits, keys):
    pages, row = -(-keys // 16), heads * dim
    return quantized._QuantAttentionArgs(batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, page_size=16, n_pages=1000, rows=batch, row_pages=pages, table_stride=pages,
                                         q_stride=(ctypes.c_int64 * 3)(tokens * row, row, dim), out_stride=(ctypes.c_int64 * 3)(tokens * row, row, dim), scale=0.125, dtype=1, bits=bits)


@pytest.mark.parametrize("batch,tokens,heads,kv_heads,dim,bits,keys", [
    (8192, 4, 8, 1, 64, 4, 1100), (4096, 4, 8, 1, 128, 4, 1100), (4000, 1, 8, 1, 64, 4, 2000), (8000, 2, 16, 2, 64, 8, 30000), (64, 4, 8, 1, 64, 4, 400), (700, 4, 8, 2, 64, 8, 200),
])
def test_uncut_sequences(lib, batch, tokens, heads, kv_heads, dim, bits, keys):
    size = lib.atk_quant_attention_workspace_bytes(args(batch, tokens, heads, kv_heads, dim, bits, keys))
    # a part is a row in f32, its maximum and its sum; at most four tiles are taken at once, of some sequences: of thousands of them none
    most = 0 if batch >= 4000 else 4 // kv_heads * batch * tokens * heads * (4 * dim + 8) + 8 * batch
    assert 0 < size <= most + 16


@pytest.mark.parametrize("batch,tokens,heads,kv_heads,dim", [(32, 1 << 17, 32, 8, 128), (1, 1 << 22, 64, 4, 128), (16, 1 << 18, 16, 16, 64)])
def test_many_rows_without_parts(lib, batch, tokens, heads, kv_heads, dim):
    assert lib.atk_quant_attention_workspace_bytes(args(batch, tokens, heads, kv_heads, dim, 4, tokens)) == 16
