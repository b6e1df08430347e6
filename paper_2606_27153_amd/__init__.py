"""MI355X-native single-GPU Muon optimizer step (DMuon, arXiv 2606.27153).

The step itself runs in the HIP library ``libmuon_mi355x.so`` built from
``csrc/``; this package is its thin Python binding (argument marshalling
only).  ``layers`` binds ``libmuon_layers.so``: the operators of the layers that
hold the stepped matrices (linear, grouped linear, layer norm, with their
backward passes).  Importing the package does not load the libraries; the first
use of a binding does, and fails loudly if its library has not been built.
"""
__all__ = ["MuonPlan", "Muon", "layers", "load_library"]


def load_library():
    from . import _lib
    return _lib.load()


def __getattr__(name):
    if name in ("MuonPlan", "Muon"):
        from . import optim
        return getattr(optim, name)
    if name == "layers":
        import importlib
        return importlib.import_module(".layers", __name__)
    raise AttributeError(name)
