"""What a decoder needs beside the selection: attention of a batch that shares a long prefix, verification of drafted
tokens, and the pages of the cache between them.

Argument marshalling only, as in binding.py (calls on plain tensors by the extension module of csrc/atk_decode_torch.cpp): the work is done by the HIP library (include/atk_decode.h), on torch's
current stream of the tensors' device, without synchronising; every call may be captured into a graph.  Shapes, types
and strides are checked here and raise; what lies on the device - page numbers, sequence numbers, lengths - is checked by
the kernels, which never follow a bad one and or a bit into the `status` tensor of the call (ATK_STATUS_*).
"""
from __future__ import annotations

import ctypes
import os

from . import binding
from .binding import ATK_BF16, ATK_F32

ATK_F16 = 2
ATK_STATUS_NO_PAGES = 1
ATK_STATUS_BAD_SEQ = 2
ATK_STATUS_BAD_PAGE = 4
ATK_STATUS_BAD_LEN = 8

_TORCH_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "_atk_decode.so")
_vp, _i64, _ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
_lib = None
_plain = None  # the extension module, from the first call on; False where it cannot be used


class _AttentionArgs(ctypes.Structure):
    _fields_ = ([(n, _vp) for n in ("q", "k", "v", "out", "lse", "page_table", "lens", "seqs", "status")]
                + [(n, _i64) for n in ("batch", "tokens", "heads", "kv_heads", "dim", "page_size", "n_pages", "rows", "row_pages", "table_stride", "prefix_len")]
                + [(n, _i64 * 3) for n in ("q_stride", "out_stride", "k_stride", "v_stride")] + [("scale", ctypes.c_double), ("dtype", ctypes.c_int32)])


class _Tables(ctypes.Structure):
    _fields_ = ([(n, _vp) for n in ("page_table", "lens", "refs", "free_pages", "n_free", "status", "work")]
                + [(n, _i64) for n in ("rows", "row_pages", "n_pages", "page_size", "work_bytes")])


def _library():
    global _lib
    if _lib is None:
        lib = binding.load_library()
        args, tables, strides = ctypes.POINTER(_AttentionArgs), ctypes.POINTER(_Tables), ctypes.POINTER(_i64)
        for name, res, types in (
                ("atk_attention_workspace_bytes", _i64, [args]),
                ("atk_shared_prefix_attention", _ci, [args, _vp, _i64, _vp]),
                ("atk_verify_workspace_bytes", _i64, [_i64] * 3),
                ("atk_verify_drafts", _ci, [_vp, strides, _vp, strides, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _ci, _vp, _vp, _vp, _i64, _vp]),
                ("atk_pages_work_bytes", _i64, [_i64]),
                ("atk_copy_pages", _ci, [_vp, _vp, _i64, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _vp]),
                ("atk_fork_sequences", _ci, [tables, _vp, _i64, _i64, _vp, _vp, _i64, _vp]),
                ("atk_append_tokens", _ci, [tables, _vp, _vp, _vp, _i64, _i64, _vp, _i64, _i64, _vp]),
                ("atk_free_sequences", _ci, [tables, _vp, _vp, _i64, _vp]),
                ("atk_compact_pages", _ci, [tables, _vp, _i64, _i64, _vp, _vp])):
            f = getattr(lib, name)
            f.restype, f.argtypes = res, types
        _lib = lib
    return _lib


def _load_plain():
    """Load (once) the extension module that marshals calls on plain tensors, as binding.py does its own.  It only saves time."""
    global _plain
    import importlib.machinery
    import importlib.util

    import torch

    lib = _library()
    try:
        loader = importlib.machinery.ExtensionFileLoader("_atk_decode", _TORCH_PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_atk_decode", loader))
        loader.exec_module(module)
        if module.torch_version != torch.__version__.split("+")[0]:
            raise ImportError("built for torch %s, this is %s" % (module.torch_version, torch.__version__))
        module.use(*(ctypes.cast(getattr(lib, "atk_" + n), _vp).value for n in ("attention_workspace_bytes", "shared_prefix_attention", "verify_workspace_bytes", "verify_drafts",
                                                                                "copy_pages", "fork_sequences", "append_tokens", "free_sequences", "compact_pages")))
    except ImportError as e:
        import warnings

        _plain = False
        warnings.warn("%s cannot be used (%s): calls take some microseconds more on the host.  `python -c 'import __graft_entry__ as g; g.build()'` at the "
                      "repository root builds it." % (_TORCH_PATH, e), RuntimeWarning, stacklevel=4)
        return False
    _plain = module
    return module


def _fast(name, *args):
    """What the extension module makes of a call: its result, or None for what it leaves to the code here."""
    module = _load_plain() if _plain is None else _plain
    if not module:
        return None
    got = getattr(module, name)(*args)
    if type(got) is int:
        binding._check(got)
    return got


def _dtype(t, what):
    import torch

    code = {torch.float32: ATK_F32, torch.bfloat16: ATK_BF16, torch.float16: ATK_F16}.get(t.dtype)
    if code is None:
        raise TypeError("%s must be float32, bfloat16 or float16" % what)
    return code


def _on_gpu(device, **tensors):
    for name, t in tensors.items():
        if t is not None and (not t.is_cuda or t.device != device):
            raise ValueError("%s must live on the GPU, all tensors on the same one" % name)


def _ints(t, shape, what):
    """A contiguous int32 tensor of that shape."""
    import torch

    if t.dtype is not torch.int32:
        raise TypeError("%s must be int32" % what)
    if tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous tensor of shape %s" % (what, shape))


def _call(device, f, *args):
    """f(*args, stream) with the device current; raises what the library refuses."""
    import torch

    index = device.index
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(device):
            return _call(device, f, *args)
    code = f(*args, torch._C._cuda_getCurrentRawStream(index))
    if code:
        binding._check(code)


def shared_prefix_attention(q, k_pages, v_pages, page_table, lens, prefix_len, seqs=None, scale=None, out=None, return_lse=False, status=None):
    """Attention of the last T tokens of each of B sequences over a paged cache whose first prefix_len keys they share.

    q (B, T, heads, dim); k_pages, v_pages (pages, page_size, kv_heads, dim), of float32, bfloat16 or float16, strided as they like but for
    a contiguous dim (a multiple of 16 bytes, up to 256 elements; pages head by head are a transposed view).  heads is a multiple
    of kv_heads.  page_table (rows, pages per row) and lens (rows) int32: row seqs[i] (int32; None: i) is sequence i's, and its
    length counts the T tokens of this call.  Token t sees the keys before lens - (T - 1 - t).  Keys before prefix_len are read
    through the first sequence's row, once for the whole batch.  scale: 1 / sqrt(dim) if None.

    Returns out (B, T, heads, dim), with return_lse also the log of the sum of exp of the scaled scores (B, T, heads) f32.
    A token that sees no key gets 0 and -inf."""
    if out is None:
        got = _fast("attention", q, k_pages, v_pages, page_table, lens, prefix_len, seqs, scale, return_lse, status)
        if got is not None:
            return got
    import torch

    if q.dim() != 4 or k_pages.dim() != 4 or v_pages.dim() != 4:
        raise ValueError("q must be (B, T, heads, dim), k_pages and v_pages (pages, page_size, kv_heads, dim)")
    code = _dtype(q, "q")
    if k_pages.dtype is not q.dtype or v_pages.dtype is not q.dtype:
        raise TypeError("q, k_pages and v_pages must be of one type")
    device = q.device
    _on_gpu(device, q=q, k_pages=k_pages, v_pages=v_pages, page_table=page_table, lens=lens, seqs=seqs, out=out, status=status)
    B, T, H, D = q.shape
    P, ps, Hk, Dk = k_pages.shape
    if v_pages.shape != k_pages.shape or Dk != D or Hk == 0 or H % Hk:
        raise ValueError("v_pages must be shaped like k_pages, with q's dim and a divisor of its heads")
    if page_table.dim() != 2 or page_table.dtype is not torch.int32 or page_table.stride(1) != 1:
        raise ValueError("page_table must be an int32 tensor (rows, pages per row) with contiguous rows")
    rows, M = page_table.shape
    _ints(lens, (rows,), "lens")
    if seqs is not None:
        _ints(seqs, (B,), "seqs")
    elif B > rows:
        raise ValueError("page_table has fewer rows than there are sequences")
    if status is not None:
        _ints(status, (1,), "status")
    if not 0 <= prefix_len <= M * ps:
        raise ValueError("prefix_len must lie between 0 and what a row of the table holds")
    if out is None:
        out = torch.empty((B, T, H, D), dtype=q.dtype, device=device)
    elif out.shape != q.shape or out.dtype is not q.dtype:
        raise ValueError("out must be shaped and typed like q")
    lse = torch.empty((B, T, H), dtype=torch.float32, device=device) if return_lse else None
    for name, t in (("q", q), ("out", out), ("k_pages", k_pages), ("v_pages", v_pages)):
        if t.numel() and t.stride(3) != 1:
            raise ValueError("the last dimension of %s must be contiguous" % name)
    if B * T * H * D == 0:
        return (out, lse) if return_lse else out
    if P * ps * M == 0:   # no key anywhere
        out.zero_()
        return (out, lse.fill_(float("-inf"))) if return_lse else out
    lib = _lib or _library()
    sq, so, sk, sv = q.stride(), out.stride(), k_pages.stride(), v_pages.stride()
    a = _AttentionArgs(q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), out.data_ptr(), lse.data_ptr() if return_lse else None, page_table.data_ptr(), lens.data_ptr(),
                       None if seqs is None else seqs.data_ptr(), None if status is None else status.data_ptr(), B, T, H, Hk, D, ps, P, rows, M,
                       page_table.stride(0) if rows > 1 else M, prefix_len, sq[:3], so[:3], sk[:3], sv[:3], D ** -0.5 if scale is None else scale, code)
    size = lib.atk_attention_workspace_bytes(a)
    if size < 0:
        binding._check(size)
    work = torch.empty((size,), dtype=torch.uint8, device=device)
    _call(device, lib.atk_shared_prefix_attention, a, work.data_ptr(), size)
    return (out, lse) if return_lse else out


def verify_drafts(target_probs, draft_tokens, draft_probs, accept_random, final_random, n_drafts=None):
    """Accepts drafted tokens by the target's probabilities and draws one more token, from given random numbers.

    target_probs (B, L + 1, vocab), draft_probs (B, L, vocab) of float32, bfloat16 or float16, vocab contiguous; draft_probs None: the
    drafts were certain.  draft_tokens (B, L) int32, accept_random (B, L) and final_random (B) float32 in [0, 1), n_drafts (B) int32
    or None for L.  Token i is accepted while accept_random * q < p, in order; the one after the last accepted is drawn from
    max(p - q, 0), or from p where every draft was accepted: the first index whose running sum exceeds final_random times the total.

    Returns accepted (B) int32 and tokens (B, L + 1) int32: the accepted ones, the drawn one, then -1."""
    got = _fast("verify", target_probs, draft_tokens, draft_probs, accept_random, final_random, n_drafts)
    if got is not None:
        return got
    import torch

    if target_probs.dim() != 3 or draft_tokens.dim() != 2:
        raise ValueError("target_probs must be (B, L + 1, vocab), draft_tokens (B, L)")
    code = _dtype(target_probs, "target_probs")
    device = target_probs.device
    _on_gpu(device, target_probs=target_probs, draft_tokens=draft_tokens, draft_probs=draft_probs, accept_random=accept_random, final_random=final_random, n_drafts=n_drafts)
    B, L = draft_tokens.shape
    V = target_probs.shape[2]
    if tuple(target_probs.shape[:2]) != (B, L + 1) or V == 0:
        raise ValueError("target_probs must be (B, L + 1, vocab) for draft_tokens (B, L)")
    _ints(draft_tokens, (B, L), "draft_tokens")
    if target_probs.stride(2) != 1 and V > 1:
        raise ValueError("the last dimension of target_probs must be contiguous")
    strides = (_i64 * 2)(*target_probs.stride()[:2])
    other = None
    if draft_probs is not None:
        if draft_probs.dtype is not target_probs.dtype:
            raise TypeError("draft_probs must be of target_probs' type")
        if tuple(draft_probs.shape) != (B, L, V) or (draft_probs.numel() and V > 1 and draft_probs.stride(2) != 1):
            raise ValueError("draft_probs must be (B, L, vocab) with a contiguous last dimension")
        other = (_i64 * 2)(*draft_probs.stride()[:2])
    for name, t, shape in (("accept_random", accept_random, (B, L)), ("final_random", final_random, (B,))):
        if t.dtype is not torch.float32:
            raise TypeError("%s must be float32" % name)
        if tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError("%s must be a contiguous tensor of shape %s" % (name, shape))
    if n_drafts is not None:
        _ints(n_drafts, (B,), "n_drafts")
    accepted = torch.empty((B,), dtype=torch.int32, device=device)
    tokens = torch.empty((B, L + 1), dtype=torch.int32, device=device)
    if B == 0:
        return accepted, tokens
    lib = _lib or _library()
    size = lib.atk_verify_workspace_bytes(B, L, V)
    if size < 0:
        binding._check(size)
    work = torch.empty((size,), dtype=torch.uint8, device=device)
    _call(device, lib.atk_verify_drafts, target_probs.data_ptr(), strides, None if other is None or L == 0 else draft_probs.data_ptr(), other, draft_tokens.data_ptr() or None,
          accept_random.data_ptr() or None, final_random.data_ptr(), None if n_drafts is None else n_drafts.data_ptr(), B, L, V, code, accepted.data_ptr(), tokens.data_ptr(),
          work.data_ptr(), size)
    return accepted, tokens


class PageTables:
    """Which pages of a cache each sequence holds, and which are free.

    page_table (rows, pages per row) int32, -1 past a sequence's pages; lens (rows) int32 tokens; refs (pages) int32, how many rows hold a page;
    free_pages (pages) int32, a stack of n_free (1,) int32 pages; status (1,) int32, to which the kernels or what they meet
    (ATK_STATUS_*).  All contiguous, on one GPU, and changed in place by fork_sequences, append_tokens, free_sequences and compact_pages;
    calls on one table belong on one stream, or have to be ordered by events."""

    def __init__(self, page_table, lens, refs, free_pages, n_free, page_size, status=None):
        import torch

        if page_table.dim() != 2:
            raise ValueError("page_table must be (rows, pages per row)")
        rows, row_pages = page_table.shape
        pages = refs.numel()
        self.device = device = page_table.device
        if status is None:
            status = torch.zeros((1,), dtype=torch.int32, device=device)
        _on_gpu(device, page_table=page_table, lens=lens, refs=refs, free_pages=free_pages, n_free=n_free, status=status)
        for name, t, shape in (("page_table", page_table, (rows, row_pages)), ("lens", lens, (rows,)), ("refs", refs, (pages,)), ("free_pages", free_pages, (pages,)),
                               ("n_free", n_free, (1,)), ("status", status, (1,))):
            _ints(t, shape, name)
        if rows < 1 or row_pages < 1 or pages < 1 or page_size < 1:
            raise ValueError("a table has a row, a page and a token in it at least")
        self.page_table, self.lens, self.refs, self.free_pages, self.n_free, self.status = page_table, lens, refs, free_pages, n_free, status
        self.page_size = page_size
        size = _library().atk_pages_work_bytes(pages)
        if size < 0:
            binding._check(size)
        self._work = torch.zeros((size,), dtype=torch.uint8, device=device)
        self._args = _Tables(page_table.data_ptr(), lens.data_ptr(), refs.data_ptr(), free_pages.data_ptr(), n_free.data_ptr(), status.data_ptr(), self._work.data_ptr(),
                             rows, row_pages, pages, page_size, size)
        self._address, self._device = ctypes.addressof(self._args), device.index

    @classmethod
    def empty(cls, pages, page_size, rows, row_pages, device="cuda"):
        """Tables of a cache that holds nothing: every page free, the lowest on top of the stack."""
        import torch

        def full(shape, v):
            return torch.full(shape, v, dtype=torch.int32, device=device)

        return cls(full((rows, row_pages), -1), full((rows,), 0), full((pages,), 0), torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=device), full((1,), pages), page_size)


def _pools(pools, device, pages, page_size, what="pools"):
    """Addresses of the pools and the bytes of a token in each."""
    token_bytes = 0
    if pages < 1 or page_size < 1:
        raise ValueError("%s must hold a page, and a token in it, at least" % what)
    for t in pools:
        if t.dim() < 2 or t.shape[0] != pages or t.shape[1] != page_size or not t.is_contiguous():
            raise ValueError("%s must be contiguous tensors (pages, page_size, ...)" % what)
        if t.device != device:
            raise ValueError("%s must live on the GPU, all tensors on the same one" % what)
        size = t.numel() // (pages * page_size) * t.element_size()
        if size < 1:
            raise ValueError("%s must hold a byte for a token at least" % what)
        if token_bytes and size != token_bytes:
            raise ValueError("%s must hold equally many bytes for a token" % what)
        token_bytes = size
    return (_vp * len(pools))(*[t.data_ptr() for t in pools]), token_bytes or 1  # (no pools: the library wants a number)


def copy_pages(src_pools, src_ids, dst_pools, dst_ids, status=None):
    """dst_pools[p][dst_ids[i]] = src_pools[p][src_ids[i]] for every pool p and every i: whole pages, between caches or within one.

    The pools are lists of contiguous tensors (pages, page_size, ...), src_ids and dst_ids int32 tensors; destinations are distinct and
    no page is both a source and a destination.  A page number out of range is passed over and reported in `status`."""
    if _fast("copy", src_pools, src_ids, dst_pools, dst_ids, status) is not None:
        return
    if len(src_pools) != len(dst_pools):
        raise ValueError("src_pools and dst_pools must be equally many")
    if src_ids.dim() != 1:
        raise ValueError("src_ids must have one dimension")
    n = src_ids.shape[0]
    device = src_ids.device
    _on_gpu(device, src_ids=src_ids, dst_ids=dst_ids, status=status)
    _ints(src_ids, (n,), "src_ids")
    _ints(dst_ids, (n,), "dst_ids")
    if status is not None:
        _ints(status, (1,), "status")
    if not src_pools or n == 0:
        return
    if src_pools[0].dim() < 2 or dst_pools[0].dim() < 2:
        raise ValueError("src_pools and dst_pools must be contiguous tensors (pages, page_size, ...)")
    for a, b in zip(src_pools, dst_pools):
        if a.dtype is not b.dtype or a.shape[1:] != b.shape[1:]:
            raise ValueError("pages of src_pools and dst_pools must have one shape and type")
    sp, dp, ps = src_pools[0].shape[0], dst_pools[0].shape[0], src_pools[0].shape[1]
    src, token_bytes = _pools(src_pools, device, sp, ps, "src_pools")
    dst, _ = _pools(dst_pools, device, dp, ps, "dst_pools")
    _call(device, (_lib or _library()).atk_copy_pages, src, dst, len(src_pools), token_bytes * ps, sp, dp, src_ids.data_ptr(), dst_ids.data_ptr(), n,
          None if status is None else status.data_ptr())


def _seqs(tables, t, n, what):
    _on_gpu(tables.device, **{what: t})
    if t.dim() != 1:
        raise ValueError("%s must have one dimension" % what)
    _ints(t, (t.shape[0] if n is None else n,), what)
    if t.shape[0] > tables._args.rows:
        raise ValueError("%s has more sequences than the table has rows" % what)
    return t.shape[0]


def fork_sequences(tables, pools, parents, children):
    """Makes row children[i] of the tables, empty until now, a copy of row parents[i] as it is at the call (so a child of the same call
    is an empty parent): whole pages are shared, a last page that is filled in part is copied, in all pools.  parents and children: int32 (n,), children distinct.  All or nothing: with too few
    free pages, or a child that holds something, nothing changes and tables.status says so."""
    if _fast("fork", tables._address, tables._device, pools, parents, children) is not None:
        return
    n = _seqs(tables, parents, None, "parents")
    _seqs(tables, children, n, "children")
    a = tables._args
    ptrs, token_bytes = _pools(pools, tables.device, a.n_pages, a.page_size)
    if n:
        _call(tables.device, _lib.atk_fork_sequences, a, ptrs, len(pools), token_bytes, parents.data_ptr(), children.data_ptr(), n)


def append_tokens(tables, pools, seqs, values):
    """Adds T tokens to each of the distinct rows seqs (int32, (n,)): values[p] (n, T, ...) goes into pools[p] behind what the rows hold.

    Takes fresh pages as they are needed, and a copy of a last page that is filled in part while other rows hold it too.  All or
    nothing: with too few free pages, or a row that is too short, nothing changes and tables.status says so."""
    if _fast("append", tables._address, tables._device, pools, seqs, values) is not None:
        return
    n = _seqs(tables, seqs, None, "seqs")
    a = tables._args
    ptrs, token_bytes = _pools(pools, tables.device, a.n_pages, a.page_size)
    if len(values) != len(pools):
        raise ValueError("values and pools must be equally many")
    if not values:
        raise ValueError("append_tokens needs a pool")
    tokens = values[0].shape[1] if values[0].dim() > 1 else 0
    for v, p in zip(values, pools):
        if v.dim() < 2 or v.shape[:2] != (n, tokens) or v.shape[2:] != p.shape[2:] or v.dtype is not p.dtype or v.device != p.device:
            raise ValueError("values must be (n, T, ...) of the pools' type, with their tokens' shape")
        if n and not v[0].is_contiguous():
            raise ValueError("a sequence's tokens in values must be contiguous")
    if n and tokens:
        at = (_vp * len(values))(*[v.data_ptr() for v in values])
        strides = (_i64 * len(values))(*[v.stride(0) * v.element_size() if n > 1 else tokens * token_bytes for v in values])
        _call(tables.device, _lib.atk_append_tokens, a, ptrs, at, strides, len(pools), token_bytes, seqs.data_ptr(), n, tokens)


def free_sequences(tables, seqs, drop=None):
    """Drops the last drop[i] tokens of row seqs[i] (all of them without `drop`) and gives back the pages that hold none of the rest,
    the lowest on top of the stack.  seqs, drop: int32 (n,), seqs distinct."""
    if _fast("free", tables._address, tables._device, seqs, drop) is not None:
        return
    n = _seqs(tables, seqs, None, "seqs")
    if drop is not None:
        _seqs(tables, drop, n, "drop")
    if n:
        _call(tables.device, _lib.atk_free_sequences, tables._args, seqs.data_ptr(), None if drop is None else drop.data_ptr(), n)


def compact_pages(tables, pools):
    """Moves the held pages to the lowest numbers, in all pools, tables and the stack.  Returns remap (pages,) int32: the new number of
    each page, -1 for those that were free - for page lists that a program keeps beside the tables."""
    got = _fast("compact", tables._address, tables._device, pools)
    if got is not None:
        return got
    import torch

    a = tables._args
    ptrs, token_bytes = _pools(pools, tables.device, a.n_pages, a.page_size)
    remap = torch.empty((a.n_pages,), dtype=torch.int32, device=tables.device)
    _call(tables.device, _lib.atk_compact_pages, a, ptrs, len(pools), token_bytes, remap.data_ptr())
    return remap
