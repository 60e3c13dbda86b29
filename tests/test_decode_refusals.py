"""The decoding operators' host side: symbols, and refusals that come before any HIP call."""
import ctypes
import os
import re

import pytest
import torch

import paper_2412_04358_amd as atk
from paper_2412_04358_amd import decode

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULLP, UNSUP, DTYPE, ALIGN, WORK, ARGS = -1, -4, -5, -7, -8, -9
FAKE = 1 << 20  # never followed: the checks come first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(atk.lib_path()):
        import __graft_entry__

        __graft_entry__.build()
    return decode._library()


def test_header_and_library_agree(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "atk_decode.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(atk_[a-z_]+)\s*\(", text))
    assert len(names) == 10
    for n in names:
        assert getattr(lib, n).argtypes is not None, n
    assert b"decoding" in lib.atk_strerror(ARGS)


def _attention(**kw):
    i3 = ctypes.c_int64 * 3
    a = dict(q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=None, page_table=FAKE, lens=FAKE, seqs=None, status=None, batch=4, tokens=1, heads=8, kv_heads=2, dim=64, page_size=16, n_pages=100,
             rows=4, row_pages=20, table_stride=20, prefix_len=100, q_stride=(512, 512, 64), out_stride=(512, 512, 64), k_stride=(2048, 128, 64), v_stride=(2048, 128, 64), scale=0.125, dtype=1)
    a.update(kw)
    for n in ("q_stride", "out_stride", "k_stride", "v_stride"):
        a[n] = i3(*a[n])
    return decode._AttentionArgs(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), ARGS), (dict(tokens=0), ARGS), (dict(heads=0), ARGS), (dict(kv_heads=3), ARGS), (dict(kv_heads=0), ARGS), (dict(page_size=0), ARGS), (dict(n_pages=0), ARGS),
    (dict(rows=3), ARGS), (dict(row_pages=0), ARGS), (dict(table_stride=19), ARGS), (dict(prefix_len=321), ARGS), (dict(prefix_len=-1), ARGS), (dict(scale=0.0), ARGS),
    (dict(scale=-1.0), ARGS), (dict(scale=float("nan")), ARGS), (dict(scale=float("inf")), ARGS), (dict(row_pages=1 << 28), ARGS), (dict(batch=1 << 31, seqs=FAKE), ARGS),
    (dict(dim=4), UNSUP), (dict(dim=60), UNSUP), (dict(dim=264), UNSUP), (dict(dim=2, dtype=0), UNSUP), (dict(dtype=3), DTYPE), (dict(dtype=-1), DTYPE),
    (dict(q_stride=(513, 512, 64)), ALIGN), (dict(k_stride=(2048, 132, 64)), ALIGN), (dict(v_stride=(-2048, 128, 64)), ARGS),
])
def test_attention_refuses(lib, kw, code):
    assert lib.atk_attention_workspace_bytes(_attention(**kw)) == code
    assert lib.atk_shared_prefix_attention(_attention(**kw), FAKE, 1 << 40, None) == code


@pytest.mark.parametrize("kw,code", [(dict(q=None), NULLP), (dict(k=None), NULLP), (dict(out=None), NULLP), (dict(page_table=None), NULLP), (dict(lens=None), NULLP), (dict(q=FAKE + 8), ALIGN),
                                     (dict(v=FAKE + 2), ALIGN), (dict(lens=FAKE + 2), ALIGN), (dict(lse=FAKE + 1), ALIGN)])
def test_attention_refuses_pointers(lib, kw, code):
    assert lib.atk_shared_prefix_attention(_attention(**kw), FAKE, 1 << 40, None) == code


def test_attention_workspace(lib):
    need = lib.atk_attention_workspace_bytes(_attention())
    assert need > 0
    assert lib.atk_shared_prefix_attention(_attention(), FAKE, need - 1, None) == WORK
    assert lib.atk_shared_prefix_attention(_attention(), FAKE + 4, need, None) == ALIGN
    assert lib.atk_shared_prefix_attention(_attention(), None, need, None) == NULLP


def _verify(lib, **kw):
    s = (ctypes.c_int64 * 2)(5000, 1000)
    a = dict(target=FAKE, ts=s, draft=FAKE, ds=s, tokens=FAKE, u=FAKE, r=FAKE, n=None, batch=2, drafts=4, vocab=1000, dtype=0, accepted=FAKE, out=FAKE, work=FAKE, bytes=1 << 30)
    a.update(kw)
    return lib.atk_verify_drafts(a["target"], a["ts"], a["draft"], a["ds"], a["tokens"], a["u"], a["r"], a["n"], a["batch"], a["drafts"], a["vocab"], a["dtype"], a["accepted"], a["out"],
                                 a["work"], a["bytes"], None)


@pytest.mark.parametrize("kw,code", [(dict(batch=0), ARGS), (dict(vocab=0), ARGS), (dict(drafts=-1), ARGS), (dict(vocab=1 << 30), ARGS), (dict(dtype=3), DTYPE), (dict(target=None), NULLP),
                                     (dict(tokens=None), NULLP), (dict(u=None), NULLP), (dict(r=None), NULLP), (dict(out=None), NULLP), (dict(work=None), NULLP), (dict(ds=None), NULLP),
                                     (dict(target=FAKE + 2), ALIGN), (dict(tokens=FAKE + 1), ALIGN), (dict(work=FAKE + 8), ALIGN), (dict(bytes=15), WORK),
                                     (dict(ts=(ctypes.c_int64 * 2)(-1, 5)), ARGS)])
def test_verify_refuses(lib, kw, code):
    assert _verify(lib, **kw) == code


def _tables(**kw):
    a = dict(page_table=FAKE, lens=FAKE, refs=FAKE, free_pages=FAKE, n_free=FAKE, status=FAKE, work=FAKE, rows=4, row_pages=8, n_pages=64, page_size=16, work_bytes=1 << 20)
    a.update(kw)
    return decode._Tables(**a)


def test_pages_refuse(lib):
    one = (ctypes.c_void_p * 1)(FAKE)
    none = (ctypes.c_void_p * 1)(None)
    stride = (ctypes.c_int64 * 1)(4096)
    for kw, code in [(dict(rows=0), ARGS), (dict(row_pages=0), ARGS), (dict(n_pages=0), ARGS), (dict(page_size=0), ARGS), (dict(row_pages=1 << 27), ARGS), (dict(lens=None), NULLP),
                     (dict(work=None), NULLP), (dict(refs=FAKE + 2), ALIGN), (dict(work=FAKE + 8), ALIGN), (dict(work_bytes=100), WORK)]:
        t = _tables(**kw)
        assert lib.atk_fork_sequences(t, one, 1, 256, FAKE, FAKE, 2, None) == code, kw
        assert lib.atk_append_tokens(t, one, one, stride, 1, 256, FAKE, 2, 1, None) == code, kw
        assert lib.atk_free_sequences(t, FAKE, None, 2, None) == code, kw
        assert lib.atk_compact_pages(t, one, 1, 256, FAKE, None) == code, kw
    t = _tables()
    assert lib.atk_fork_sequences(t, one, 1, 256, FAKE, FAKE, 5, None) == ARGS       # more children than rows
    assert lib.atk_fork_sequences(t, one, 1, 256, None, FAKE, 2, None) == NULLP
    assert lib.atk_fork_sequences(t, none, 1, 256, FAKE, FAKE, 2, None) == NULLP
    assert lib.atk_fork_sequences(t, one, 1, 0, FAKE, FAKE, 2, None) == ARGS
    assert lib.atk_append_tokens(t, one, none, stride, 1, 256, FAKE, 2, 1, None) == NULLP
    assert lib.atk_append_tokens(t, one, one, None, 1, 256, FAKE, 2, 1, None) == NULLP
    assert lib.atk_append_tokens(t, one, one, (ctypes.c_int64 * 1)(-4), 1, 256, FAKE, 2, 1, None) == ARGS
    assert lib.atk_append_tokens(t, one, one, stride, 1, 256, FAKE, 2, -1, None) == ARGS
    assert lib.atk_free_sequences(t, FAKE + 2, None, 2, None) == ALIGN
    assert lib.atk_compact_pages(t, one, 1, 256, None, None) == NULLP
    assert lib.atk_copy_pages(one, one, 1, 4096, 8, 8, None, FAKE, 2, None, None) == NULLP
    assert lib.atk_copy_pages(one, none, 1, 4096, 8, 8, FAKE, FAKE, 2, None, None) == NULLP
    assert lib.atk_copy_pages(one, one, 1, 4096, 0, 8, FAKE, FAKE, 2, None, None) == ARGS
    assert lib.atk_copy_pages(one, one, 1, 4096, 8, 8, FAKE, FAKE, -1, None, None) == ARGS
    # nothing to do
    assert lib.atk_fork_sequences(t, one, 1, 256, FAKE, FAKE, 0, None) == 0
    assert lib.atk_append_tokens(t, one, one, stride, 1, 256, FAKE, 0, 3, None) == 0
    assert lib.atk_free_sequences(t, FAKE, None, 0, None) == 0
    assert lib.atk_copy_pages(one, one, 1, 4096, 8, 8, FAKE, FAKE, 0, None, None) == 0


def test_python_refuses_tensors_elsewhere():
    q = torch.zeros((2, 1, 4, 64))
    kv = torch.zeros((4, 16, 2, 64))
    table, lens = torch.zeros((2, 4), dtype=torch.int32), torch.ones((2,), dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        atk.shared_prefix_attention(q, kv, kv, table, lens, 0)
    with pytest.raises(ValueError, match="must be"):
        atk.shared_prefix_attention(q[0], kv, kv, table, lens, 0)
    with pytest.raises(TypeError, match="float32"):
        atk.shared_prefix_attention(q.double(), kv, kv, table, lens, 0)
    with pytest.raises(TypeError, match="one type"):
        atk.shared_prefix_attention(q, kv.half(), kv, table, lens, 0)
    p = torch.zeros((2, 4, 10))
    with pytest.raises(ValueError, match="GPU"):
        atk.verify_drafts(p, torch.zeros((2, 3), dtype=torch.int32), None, torch.zeros((2, 3)), torch.zeros((2,)))
    with pytest.raises(ValueError, match="GPU"):
        atk.PageTables.empty(8, 16, 2, 4, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        atk.copy_pages([kv], lens, [kv], lens)
    with pytest.raises(ValueError, match="equally many"):
        atk.copy_pages([kv], lens, [], lens)
