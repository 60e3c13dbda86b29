"""A cache in few bits beside that of decode.py: tokens are quantised as they are appended, read back, and attended to.

A pool is a contiguous uint8 tensor (pages, page_size, quantized_token_bytes(kv_heads, dim, bits)): rows of e2m1 (bits 4) or e4m3 (bits 8) codes with
a power of two for each 32 elements of a head (include/atk_quant.h has the layout and the rounding).  fork_sequences, compact_pages and copy_pages move such pools as
they are.  Argument marshalling only (calls on plain tensors by the extension module of csrc/atk_quant_torch.cpp), with decode.py's conventions: torch's current stream of the tensors' device, no synchronising, every call may be captured.
"""
from __future__ import annotations

import ctypes

from . import binding, decode, plain
from .decode import _call, _ci, _dtype, _i64, _ints, _on_gpu, _seqs, _vp

_lib = None


class _QuantAttentionArgs(ctypes.Structure):
    _fields_ = ([(n, _vp) for n in ("q", "k", "v", "out", "lse", "page_table", "lens", "seqs", "status")]
                + [(n, _i64) for n in ("batch", "tokens", "heads", "kv_heads", "dim", "page_size", "n_pages", "rows", "row_pages", "table_stride")]
                + [(n, _i64 * 3) for n in ("q_stride", "out_stride")] + [("scale", ctypes.c_double), ("dtype", ctypes.c_int32), ("bits", ctypes.c_int32)])


def _library():
    global _lib
    if _lib is None:
        lib = decode._library()
        args, tables = ctypes.POINTER(_QuantAttentionArgs), ctypes.POINTER(decode._Tables)
        for name, res, types in (
                ("atk_quant_token_bytes", _i64, [_i64, _i64, _ci]),
                ("atk_append_quantized", _ci, [tables, _vp, _vp, _vp, _i64, _i64, _i64, _ci, _ci, _vp, _i64, _i64, _vp]),
                ("atk_read_quantized", _ci, [tables, _vp, _vp, _i64, _i64, _i64, _ci, _ci, _vp, _vp, _i64, _i64, _vp]),
                ("atk_quant_attention_workspace_bytes", _i64, [args]),
                ("atk_quant_attention", _ci, [args, _vp, _i64, _vp])):
            f = getattr(lib, name)
            f.restype, f.argtypes = res, types
        _lib = lib
    return _lib


def quantized_token_bytes(kv_heads, dim, bits=4):
    """Bytes of a token's row in a pool: kv_heads * (dim * bits / 8 + dim / 32), in whole 16.  dim: a multiple of 32, up to 256; bits: 4 or 8."""
    size = (_lib or _library()).atk_quant_token_bytes(kv_heads, dim, bits)
    if size < 0:
        binding._check(size)
    return size


def _pool(t, what, device, pages, page_size, token_bytes):
    import torch

    if t.dtype is not torch.uint8:
        raise TypeError("%s must be uint8" % what)
    if tuple(t.shape) != (pages, page_size, token_bytes) or not t.is_contiguous():
        raise ValueError("%s must be contiguous, of shape %s" % (what, (pages, page_size, token_bytes)))
    if t.device != device:
        raise ValueError("%s must live on the GPU, all tensors on the same one" % what)
    return t.data_ptr()


def append_quantized(tables, pools, seqs, values, bits=4):
    """append_tokens for quantised pools: adds T tokens to each of the distinct rows seqs (int32, (n,)); values[p] (n, T, kv_heads, dim), of one of float32, bfloat16
    and float16, is quantised as it goes into pools[p] behind what the rows hold.  A token's values are contiguous, tokens and sequences strided as they like (by whole 16 bytes).

    Fresh pages, copies of shared pages, and all or nothing are as for append_tokens."""
    if plain.call("append", tables._address, tables._device, pools, seqs, values, bits) is not None:
        return
    n = _seqs(tables, seqs, None, "seqs")
    a = tables._args
    if len(values) != len(pools):
        raise ValueError("values and pools must be equally many")
    if not values:
        raise ValueError("append_quantized needs a pool")
    first = values[0]
    if first.dim() != 4:
        raise ValueError("values must be (n, T, kv_heads, dim)")
    code = _dtype(first, "values")
    _, tokens, heads, dim = first.shape
    size = quantized_token_bytes(heads, dim, bits)
    ptrs = [_pool(p, "pools", tables.device, a.n_pages, a.page_size, size) for p in pools]
    strides = []
    for v in values:
        if v.shape != (n, tokens, heads, dim) or v.dtype is not first.dtype or v.device != tables.device:
            raise ValueError("values must be (n, T, kv_heads, dim) of one type, on the tables' GPU")
        s = v.stride()
        if n and tokens and (s[3] != 1 or (heads > 1 and s[2] != dim)):
            raise ValueError("a token's values must be contiguous")
        strides += [s[0] * v.element_size(), s[1] * v.element_size()]
    if n and tokens:
        k = len(values)
        _call(tables.device, _library().atk_append_quantized, a, (_vp * k)(*ptrs), (_vp * k)(*[v.data_ptr() for v in values]), (_i64 * (2 * k))(*strides), k, heads, dim, bits, code,
              seqs.data_ptr(), n, tokens)


def read_quantized(tables, pools, seqs, starts, tokens, kv_heads, dim, bits=4, dtype=None):
    """Tokens starts[i], starts[i] + 1, ... of rows seqs[i] (int32, (n,); a row may come more than once), `tokens` of each, out of quantised pools; starts None: from 0 on.

    Returns for each pool a tensor (n, tokens, kv_heads, dim) of `dtype` (bfloat16 if None; float32, bfloat16 or float16), 0 where a row has no such token."""
    import torch

    dtype = dtype or torch.bfloat16
    code = {torch.float32: decode.ATK_F32, torch.bfloat16: decode.ATK_BF16, torch.float16: decode.ATK_F16}.get(dtype)
    if code is None:
        raise TypeError("dtype must be float32, bfloat16 or float16")
    got = plain.call("read", tables._address, tables._device, pools, seqs, starts, tokens, kv_heads, dim, bits, code)
    if got is not None:
        return got
    _on_gpu(tables.device, seqs=seqs, starts=starts)
    if seqs.dim() != 1:
        raise ValueError("seqs must have one dimension")
    n = seqs.shape[0]
    _ints(seqs, (n,), "seqs")
    if starts is not None:
        _ints(starts, (n,), "starts")
    if tokens < 0:
        raise ValueError("tokens must not be negative")
    a = tables._args
    size = quantized_token_bytes(kv_heads, dim, bits)
    ptrs = [_pool(p, "pools", tables.device, a.n_pages, a.page_size, size) for p in pools]
    outs = [torch.empty((n, tokens, kv_heads, dim), dtype=dtype, device=tables.device) for _ in pools]
    if n and tokens and outs:
        k = len(outs)
        _call(tables.device, _library().atk_read_quantized, a, (_vp * k)(*ptrs), (_vp * k)(*[o.data_ptr() for o in outs]), k, kv_heads, dim, bits, code, seqs.data_ptr(),
              None if starts is None else starts.data_ptr(), n, tokens)
    return outs


def quantized_attention(q, k_pages, v_pages, page_table, lens, kv_heads, bits=4, seqs=None, scale=None, out=None, return_lse=False, status=None):
    """Attention of the last T tokens of each of B sequences over quantised pools.

    q (B, T, heads, dim) of float32, bfloat16 or float16, strided as it likes (by whole 16 bytes) but for a contiguous dim, and so is out; heads is a multiple of kv_heads, dim of 32, up to 256.
    k_pages, v_pages (pages, page_size, quantized_token_bytes(kv_heads, dim, bits)) uint8.  page_table (rows, pages per row) and lens (rows) int32: row seqs[i]
    (int32; None: i) is sequence i's, and its length counts the T tokens of this call.  Token t sees the keys before lens - (T - 1 - t).  scale: 1 / sqrt(dim) if None.

    Returns out (B, T, heads, dim), with return_lse also the log of the sum of exp of the scaled scores (B, T, heads) f32: what shared_prefix_attention gives on the
    values that read_quantized gives in q's type.  A token that sees no key gets 0 and -inf.  Autograd sees none of it: results require no gradient, whatever q does."""
    if out is None:
        got = plain.call("attention", q, k_pages, v_pages, page_table, lens, kv_heads, bits, seqs, scale, return_lse, status)
        if got is not None:
            return got
    import torch

    if q.dim() != 4 or k_pages.dim() != 3:
        raise ValueError("q must be (B, T, heads, dim), k_pages and v_pages (pages, page_size, bytes)")
    code = _dtype(q, "q")
    device = q.device
    _on_gpu(device, q=q, k_pages=k_pages, v_pages=v_pages, page_table=page_table, lens=lens, seqs=seqs, out=out, status=status)
    B, T, H, D = q.shape
    size = quantized_token_bytes(kv_heads, D, bits)
    P, ps = k_pages.shape[:2]
    if H % kv_heads:
        raise ValueError("q's heads must be a multiple of kv_heads")
    k = _pool(k_pages, "k_pages", device, P, ps, size)
    v = _pool(v_pages, "v_pages", device, P, ps, size)
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
    if out is None:
        out = torch.empty((B, T, H, D), dtype=q.dtype, device=device)
    elif out.shape != q.shape or out.dtype is not q.dtype:
        raise ValueError("out must be shaped and typed like q")
    lse = torch.empty((B, T, H), dtype=torch.float32, device=device) if return_lse else None
    for name, t in (("q", q), ("out", out)):
        if t.numel() and t.stride(3) != 1:
            raise ValueError("the last dimension of %s must be contiguous" % name)
    if B * T * H == 0:
        return (out, lse) if return_lse else out
    if P * ps * M == 0:   # no key anywhere
        out.zero_()
        return (out, lse.fill_(float("-inf"))) if return_lse else out
    sq, so = q.stride(), out.stride()
    a = _QuantAttentionArgs(q.data_ptr(), k, v, out.data_ptr(), lse.data_ptr() if return_lse else None, page_table.data_ptr(), lens.data_ptr(),
                            None if seqs is None else seqs.data_ptr(), None if status is None else status.data_ptr(), B, T, H, kv_heads, D, ps, P, rows, M,
                            page_table.stride(0) if rows > 1 else M, sq[:3], so[:3], D ** -0.5 if scale is None else scale, code, bits)
    bytes_ = _lib.atk_quant_attention_workspace_bytes(a)
    if bytes_ < 0:
        binding._check(bytes_)
    work = torch.empty((bytes_,), dtype=torch.uint8, device=device)
    _call(device, _lib.atk_quant_attention, a, work.data_ptr(), bytes_)
    torch.autograd.graph.increment_version(out)  # (autograd may have saved it)
    return (out, lse) if return_lse else out
