"""B200-native step executor for the Sparbit allgather (arXiv 2109.08751).

The package is a thin ctypes binding over libsparbit_b200.so (see include/sparbit.h for the
collective and include/sparbit_train.h for the training operators next to it).  Build the library
in-tree with `python -m paper_2109_08751_b200.build`.

The binding is loaded on first use of any of its names, so that the build module can be imported
before the library exists.  There is no fallback: using the package without the built library
raises ImportError.
"""
import importlib

_binding = None
_train = None


def __getattr__(name):
    global _binding, _train
    if name.startswith("__"):
        raise AttributeError(name)
    if name in ("build", "binding", "multi", "train"):  # submodules
        return importlib.import_module("." + name, __name__)
    if _binding is None:
        _binding = importlib.import_module(".binding", __name__)
        _train = importlib.import_module(".train", __name__)
    for module in (_binding, _train):
        if hasattr(module, name):
            value = globals()[name] = getattr(module, name)  # found directly from now on
            return value
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
