"""The decoding operators' host side: sizes at the ends of what the kernels count in, refused before any HIP call."""
import ctypes

import pytest

import paper_2412_04358_amd as atk
from paper_2412_04358_amd import decode

ARGS = -9
FAKE = 1 << 20  # never followed: the checks come first


@pytest.fixture(scope="module")
def lib():
    import os

    if not os.path.exists(atk.lib_path()):
        import __graft_entry__

        __graft_entry__.build()
    return decode._library()


def _tables(**kw):
    a = dict(page_table=FAKE, lens=FAKE, refs=FAKE, free_pages=FAKE, n_free=FAKE, status=FAKE, work=FAKE, rows=1 << 20, row_pages=1 << 20, n_pages=64, page_size=1, work_bytes=1 << 20)
    a.update(kw)
    return decode._Tables(**a)


@pytest.mark.parametrize("n,tokens,page_size", [(2048, 1 << 20, 1), (1 << 20, 2047, 1), (1 << 20, 2047 * 16, 16), (1 << 20, 2046 * 16 + 1, 16), (3, 1 << 30, 1)])
def test_append_of_more_pages_than_are_counted(lib, n, tokens, page_size):
    # (the values may be one sequence's for all: a stride of 0)
    one, stride = (ctypes.c_void_p * 1)(FAKE), (ctypes.c_int64 * 1)(0)
    t = _tables(page_size=page_size, row_pages=(1 << 30) // page_size if tokens >> 20 else 1 << 16)
    assert lib.atk_append_tokens(t, one, one, stride, 1, 256, FAKE, n, tokens, None) == ARGS


def _attention(**kw):
    i3 = ctypes.c_int64 * 3
    a = dict(q=FAKE, k=FAKE, v=FAKE, out=FAKE, page_table=FAKE, lens=FAKE, batch=1, tokens=1, heads=64, kv_heads=64, dim=64, page_size=16, n_pages=100, rows=1 << 26, row_pages=20,
             table_stride=20, prefix_len=0, scale=0.125, dtype=1)
    a.update(kw)
    H, D = a["heads"], a["dim"]
    for n in ("q_stride", "out_stride"):
        a[n] = i3(a["tokens"] * H * D, H * D, D)
    for n in ("k_stride", "v_stride"):
        a[n] = i3(16 * a["kv_heads"] * D, a["kv_heads"] * D, D)
    return decode._AttentionArgs(**a)


@pytest.mark.parametrize("kw,fits", [
    (dict(batch=1 << 18), False), (dict(batch=(1 << 18) - 1), True),                # one workgroup a sequence and head, 2^24 of them
    (dict(batch=1 << 20, kv_heads=1), False), (dict(batch=1 << 19, kv_heads=1, tokens=2), False), (dict(batch=(1 << 20) - 1, kv_heads=1), True),      # 2^26 rows to join
    (dict(batch=1, tokens=1 << 20, kv_heads=8, row_pages=1 << 17, table_stride=1 << 17), False), (dict(batch=1, tokens=(1 << 20) - 1, kv_heads=8, row_pages=1 << 17, table_stride=1 << 17), True),
    (dict(batch=1 << 20, kv_heads=64, heads=64, prefix_len=320, dtype=0), False),
])
def test_attention_of_more_rows_than_a_launch_takes(lib, kw, fits):
    need = lib.atk_attention_workspace_bytes(_attention(**kw))
    assert need > 0 if fits else need == ARGS
    if not fits:
        assert lib.atk_shared_prefix_attention(_attention(**kw), FAKE, 1 << 60, None) == ARGS


@pytest.mark.parametrize("batch,vocab,dtype,fits", [(1 << 22, 8, 0, False), ((1 << 22) - 1, 8, 0, True), (1 << 22, 65536, 1, False), (1 << 22, 65536, 0, False), (1 << 20, 32769, 0, True),
                                                    (1 << 20, 128256, 1, False), (1 << 24, 4, 1, False)])
def test_verification_of_more_requests_than_a_launch_takes(lib, batch, vocab, dtype, fits):
    s = (ctypes.c_int64 * 2)(0, 0)

    def call(work_bytes):
        return lib.atk_verify_drafts(FAKE, s, FAKE, s, FAKE, FAKE, FAKE, None, batch, 1, vocab, dtype, FAKE, FAKE, FAKE, work_bytes, None)

    # (one that fits is refused for its workspace, behind the sizes)
    assert call(0) == (-8 if fits else ARGS)
    if fits:
        assert lib.atk_verify_workspace_bytes(batch, 1, vocab) > 0


def test_pages_of_more_sequences_than_a_launch_takes(lib):
    one, stride = (ctypes.c_void_p * 1)(FAKE), (ctypes.c_int64 * 1)(0)
    t = _tables(rows=1 << 25, row_pages=2, page_size=16)
    for n in (1 << 24, 1 << 25):
        assert lib.atk_fork_sequences(t, one, 1, 256, FAKE, FAKE, n, None) == ARGS
        assert lib.atk_append_tokens(t, one, one, stride, 1, 256, FAKE, n, 1, None) == ARGS
        assert lib.atk_free_sequences(t, FAKE, None, n, None) == ARGS
    # (one less is refused for its addresses only)
    assert lib.atk_free_sequences(t, FAKE + 2, None, (1 << 24) - 1, None) == -7


@pytest.mark.parametrize("scale,fits", [(5e-46, False), (1e-60, False), (5e-324, False), (1e-40, False), (1.1754e-38, False), (1.18e-38, True), (1e-6, True), (1e30, True), (1.1e30, False)])
def test_scales_that_f32_does_not_hold(lib, scale, fits):
    a = _attention(batch=4, scale=scale)
    assert (lib.atk_attention_workspace_bytes(a) > 0) is fits
    if not fits:
        assert lib.atk_attention_workspace_bytes(a) == ARGS and lib.atk_shared_prefix_attention(a, FAKE, 1 << 40, None) == ARGS


def test_strides_of_single_elements_are_not_used(lib):
    i3 = ctypes.c_int64 * 3
    odd = dict(batch=1, tokens=1, heads=1, kv_heads=1, n_pages=1, page_size=1, rows=1, prefix_len=0)
    for name in ("q_stride", "out_stride", "k_stride", "v_stride"):
        for many, size in enumerate((("batch", "tokens", "heads") if name[0] in "qo" else ("n_pages", "page_size", "kv_heads"))):
            a = _attention(**odd)
            setattr(a, name, i3(*[65 if i == many else 64 for i in range(3)]))
            assert lib.atk_attention_workspace_bytes(a) > 0, (name, size)
            setattr(a, size, 2)
            a.heads, a.rows = 2 if size in ("heads", "kv_heads") else 1, 2
            if size != "heads":
                a.q_stride = i3(64, 64, 64) if name != "q_stride" else a.q_stride
            assert lib.atk_attention_workspace_bytes(a) == -7, (name, size)


def test_strides_that_offsets_of_16_bytes_reach(lib):
    # 300 sequences of 8 heads on 2 of 128: the plan of many rows up to pages of 2^34 elements in all and tokens below 2^28, and 2^34 in a page; that of few rows past it
    i3 = ctypes.c_int64 * 3

    def need(page, token, which="k_stride", n_pages=8):
        a = _attention(batch=300, heads=8, kv_heads=2, dim=128, page_size=256, n_pages=n_pages, rows=300, row_pages=8, table_stride=8, prefix_len=7 * 256)
        a.k_stride = a.v_stride = i3(256 * 256, 256, 128)
        setattr(a, which, i3(page, token, 128))
        return lib.atk_attention_workspace_bytes(a)

    near = need(256 * 256, 256)
    for which in ("k_stride", "v_stride"):
        assert need(1 << 31, 256, which) == near and need((1 << 31) + 8, 256, which) != near
        assert need(1 << 30, 256, which, 16) == near and need((1 << 30) + 8, 256, which, 16) != near
        assert need(256, (1 << 26), which) == near and need(256, (1 << 26) + 8, which) != near
