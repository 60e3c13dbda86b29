"""The extension module of csrc/atk_quant_torch.cpp, which marshals calls on plain tensors for quantized.py and scores.py.  It only saves time."""
from __future__ import annotations

import ctypes
import os

from . import binding

_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "_atk_quant.so")
_NAMES = ("quant_token_bytes", "append_quantized", "read_quantized", "quant_attention_workspace_bytes", "quant_attention", "token_logprobs_workspace_bytes", "token_logprobs", "token_logprobs_grad")
_module = None  # from the first call on; False where it cannot be used


def _load():
    """Load it (once), as decode.py does its own."""
    global _module
    import importlib.machinery
    import importlib.util

    import torch

    lib = binding.load_library()
    try:
        loader = importlib.machinery.ExtensionFileLoader("_atk_quant", _PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_atk_quant", loader))
        loader.exec_module(module)
        if module.torch_version != torch.__version__.split("+")[0]:
            raise ImportError("built for torch %s, this is %s" % (module.torch_version, torch.__version__))
        module.use(*(ctypes.cast(getattr(lib, "atk_" + n), ctypes.c_void_p).value for n in _NAMES))
    except ImportError as e:
        import warnings

        _module = False
        warnings.warn("%s cannot be used (%s): calls take some microseconds more on the host.  `python -c 'import __graft_entry__ as g; g.build()'` at the "
                      "repository root builds it." % (_PATH, e), RuntimeWarning, stacklevel=5)
        return False
    _module = module
    return module


def call(name, *args):
    """What the extension module makes of a call: its result, or None for what it leaves to the code in Python."""
    module = _load() if _module is None else _module
    if not module:
        return None
    got = getattr(module, name)(*args)
    if type(got) is int:
        binding._check(got)
    return got
