"""ctypes binding of libmuon_layers.so (the C ABI declared in
include/muon_layers.h).  Argument marshalling only; ``load()`` raises if the
library has not been built -- there is no fallback path."""
from __future__ import annotations

import ctypes
import os
import threading

from ._lib import MUON_OK, MuonError

LIB_NAME = "libmuon_layers.so"
LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), LIB_NAME)

# muon_activation
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
MUON_GROUPED_MAX_EXPERTS = 256

_P, _I32, _I64, _SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
_PP = ctypes.POINTER(ctypes.c_void_p)
_PSZ = ctypes.POINTER(ctypes.c_size_t)
_ST = ctypes.c_int

# name -> (restype, argtypes); every function declared in include/muon_layers.h
SIGNATURES = {
    "muon_linear_forward": (_ST, [_P, _I64, _P, _I64, _I32, _P, _P, _I64, _P, _I64, _P, _I64, _I64, _I64, _I64,
                                  _I32, _I32, _P, _SZ, _P]),
    "muon_linear_backward": (_ST, [_P, _I64, _P, _I64, _P, _I64, _I32, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _I64,
                                   _I64, _I32, _I32, _P, _SZ, _P]),
    "muon_linear_workspace_bytes": (_ST, [_I64, _I64, _I64, _I32, _I32, _I32, _PSZ]),
    "muon_grouped_linear_forward": (_ST, [_P, _I64, _PP, _I64, _I32, _P, _I32, _P, _I64, _I64, _I64, _I64, _I32,
                                          _P, _SZ, _P]),
    "muon_grouped_linear_backward": (_ST, [_P, _I64, _P, _I64, _PP, _I64, _I32, _P, _I32, _P, _I64, _PP, _I64, _I64,
                                           _I64, _I64, _I32, _P, _SZ, _P]),
    "muon_grouped_linear_workspace_bytes": (_ST, [_I64, _I64, _I64, _I32, _I32, _I32, _PSZ]),
    "muon_layer_norm_forward": (_ST, [_P, _I64, _P, _P, _P, _I64, _P, _P, _I64, _I64, ctypes.c_float, _I32, _I32,
                                      _P]),
    "muon_layer_norm_backward": (_ST, [_P, _I64, _P, _I64, _P, _P, _P, _P, _I64, _P, _P, _I64, _I64, _I32, _I32, _P,
                                       _SZ, _P]),
    "muon_layer_norm_workspace_bytes": (_ST, [_I64, _I64, _PSZ]),
    "muon_layers_last_error": (ctypes.c_char_p, []),
}

_lock = threading.Lock()
_lib = None


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


def check(status: int) -> None:
    if status != MUON_OK:
        raise MuonError(status, load().muon_layers_last_error().decode())
