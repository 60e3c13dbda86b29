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
