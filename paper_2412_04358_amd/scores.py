"""The scores of tokens that a decoder chose: their log probabilities with the entropy and the likeliest alternatives, and the gradient of the first two.

Argument marshalling only (calls on plain tensors by the extension module of csrc/atk_quant_torch.cpp), with decode.py's conventions (include/atk_scores.h): torch's current stream of the tensors' device, no synchronising, every call may be captured.
There is no autograd here: the gradient is a call of its own.
"""
from __future__ import annotations

from . import binding, decode, plain
from .decode import _call, _ci, _dtype, _i64, _ints, _on_gpu, _vp

_lib = None


def _library():
    global _lib
    if _lib is None:
        import ctypes

        lib = decode._library()
        strides = ctypes.POINTER(_i64)
        for name, res, types in (
                ("atk_token_logprobs_workspace_bytes", _i64, [_i64] * 4 + [_ci]),
                ("atk_token_logprobs", _ci, [_vp, strides, _vp, _i64, _i64, _i64, _i64, _ci] + [_vp] * 6 + [_i64, _vp]),
                ("atk_token_logprobs_grad", _ci, [_vp, strides] + [_vp] * 5 + [_i64, _i64, _i64, _ci, _vp, strides, _vp])):
            f = getattr(lib, name)
            f.restype, f.argtypes = res, types
        _lib = lib
    return _lib


def _rows(t, what):
    """(type, strides) of logits or of their gradient."""
    code = _dtype(t, what)
    if t.dim() != 3:
        raise ValueError("%s must be (B, T, vocab)" % what)
    if t.numel() and t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError("the last dimension of %s must be contiguous" % what)
    return code, (_i64 * 2)(*t.stride()[:2])


def _floats(t, shape, what):
    import torch

    if t.dtype is not torch.float32:
        raise TypeError("%s must be float32" % what)
    if tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous tensor of shape %s" % (what, shape))
    return t.data_ptr()


def token_logprobs(logits, tokens, top=0):
    """Log probabilities of given tokens under softmax(logits), with the entropy of the distribution and its `top` (up to 32) likeliest tokens.

    logits (B, T, vocab) of float32, bfloat16 or float16, strided as they like but for a contiguous vocab; tokens (B, T) int32, outside of the vocabulary where there is none
    (its log probability is -inf).  Returns logprobs (B, T), entropy (B, T), lse (B, T), the log of the sum of exp of the logits, top_logprobs (B, T, top), all f32, and
    top_tokens (B, T, top) int32: the likeliest first, equally likely ones by their numbers.  None of these requires a gradient, also where logits do: token_logprobs_grad is theirs."""
    got = plain.call("logprobs", logits, tokens, top)
    if got is not None:
        return got
    import torch

    code, strides = _rows(logits, "logits")
    device = logits.device
    _on_gpu(device, logits=logits, tokens=tokens)
    B, T, V = logits.shape
    _ints(tokens, (B, T), "tokens")
    if V == 0 or not 0 <= top <= min(32, V):
        raise ValueError("there must be a vocabulary, and top lie between 0 and 32 and not past it")
    logprobs, entropy, lse = torch.empty((3, B, T), dtype=torch.float32, device=device).unbind(0)
    top_logprobs = torch.empty((B, T, top), dtype=torch.float32, device=device)
    top_tokens = torch.empty((B, T, top), dtype=torch.int32, device=device)
    if B * T:
        lib = _lib or _library()
        size = lib.atk_token_logprobs_workspace_bytes(B, T, V, top, code)
        if size < 0:
            binding._check(size)
        work = torch.empty((size,), dtype=torch.uint8, device=device)
        _call(device, lib.atk_token_logprobs, logits.data_ptr(), strides, tokens.data_ptr(), B, T, V, top, code, logprobs.data_ptr(), entropy.data_ptr(), lse.data_ptr(),
              top_logprobs.data_ptr() or None, top_tokens.data_ptr() or None, work.data_ptr(), size)
    return logprobs, entropy, lse, top_logprobs, top_tokens


def token_logprobs_grad(logits, tokens, lse, entropy, grad_logprobs, grad_entropy=None, out=None):
    """Gradient with respect to the logits of sum(grad_logprobs * logprobs) + sum(grad_entropy * entropy) of token_logprobs(logits, tokens).

    lse, entropy as that call gave them (entropy may be None where grad_entropy is), grad_logprobs (None: 0) and grad_entropy (B, T) float32.  Returns a tensor like logits, in `out` if given:
    of their shape and type, strided as it likes but for a contiguous vocab and rows that do not overlap, the logits themselves if they are not needed any more.  It is what logits.backward() takes."""
    if out is None:
        got = plain.call("grad", logits, tokens, lse, entropy, grad_logprobs, grad_entropy)
        if got is not None:
            return got
    import torch

    code, strides = _rows(logits, "logits")
    device = logits.device
    _on_gpu(device, logits=logits, tokens=tokens, lse=lse, entropy=entropy, grad_logprobs=grad_logprobs, grad_entropy=grad_entropy, out=out)
    B, T, V = logits.shape
    _ints(tokens, (B, T), "tokens")
    if grad_entropy is not None and entropy is None:
        raise ValueError("the gradient of the entropy needs the entropy")
    ptrs = [None if t is None else _floats(t, (B, T), what) for what, t in (("lse", lse), ("entropy", entropy), ("grad_logprobs", grad_logprobs), ("grad_entropy", grad_entropy))]
    if out is None:
        out = torch.empty((B, T, V), dtype=logits.dtype, device=device)
    elif out.shape != logits.shape or out.dtype is not logits.dtype:
        raise ValueError("out must be shaped and typed like logits")
    _, out_strides = _rows(out, "out")
    if B * T * V:
        _call(device, (_lib or _library()).atk_token_logprobs_grad, logits.data_ptr(), strides, tokens.data_ptr(), *ptrs, B, T, V, code, out.data_ptr(), out_strides)
        torch.autograd.graph.increment_version(out)  # (autograd may have saved it, the logits above all)
    return out
