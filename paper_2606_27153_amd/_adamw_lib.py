"""ctypes binding of libmuon_adamw.so (the C ABI declared in
include/muon_adamw.h), and of the extension that reads its tensors.  Argument
marshalling only; ``load()`` and ``tensors()`` raise if their library has not been
built -- there is no fallback path."""
from __future__ import annotations

import ctypes
import os
import threading

from ._lib import MUON_OK, MuonError

LIB_NAME = "libmuon_adamw.so"
LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), LIB_NAME)
MUON_ADAMW_BLOCK = 256

_P, _I32, _I64, _D = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
_ST = ctypes.c_int


class muon_adamw_tensor(ctypes.Structure):
    _fields_ = [("param", _P), ("grad", _P), ("exp_avg", _P), ("exp_avg_sq", _P), ("bases", _P), ("n", _I64),
                ("step", _I64), ("param_dtype", _I32), ("grad_dtype", _I32)]


class muon_adamw_opts(ctypes.Structure):
    _fields_ = [("lr", _D), ("beta1", _D), ("beta2", _D), ("eps", _D), ("weight_decay", _D), ("state_bits", _I32),
                ("seed", ctypes.c_uint32)]


# name -> (restype, argtypes); every function declared in include/muon_adamw.h
SIGNATURES = {
    "muon_adamw_step": (_ST, [_P, _I32, ctypes.POINTER(muon_adamw_opts), _P]),
    "muon_adamw_state_values": (_ST, [_P, _P, _P, _I64, _P, _P, _P]),
    "muon_adamw_last_error": (ctypes.c_char_p, []),
}

_lock = threading.Lock()
_lib = None
_tensors = None
_written = None


def load(path: str = LIB_PATH):
    """Loads the HIP library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(path):
            raise RuntimeError(
                f"{LIB_NAME} not found at {path}; build it first with "
                f"`python -m paper_2606_27153_amd.build` (there is no fallback path)")
        lib = ctypes.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
        return lib


def tensors():
    """adamw_tensors(params, grads, states, steps) of csrc/adamw/binding.cpp."""
    global _tensors, _written
    if _tensors is None:
        import torch  # noqa: F401  (whose libraries the extension is linked to)
        try:
            from ._adamw_binding import adamw_tensors, adamw_written
        except ImportError as e:
            raise RuntimeError(f"_adamw_binding.so cannot be loaded ({e}); build it first with "
                               f"`python -m paper_2606_27153_amd.build` (there is no fallback path)") from e
        _written = adamw_written
        _tensors = adamw_tensors
    return _tensors


def written(params, grads, states) -> None:
    """adamw_written of csrc/adamw/binding.cpp."""
    if _written is None:
        tensors()
    _written(params, grads, states)


def check(status: int) -> None:
    if status != MUON_OK:
        raise MuonError(status, load().muon_adamw_last_error().decode())
