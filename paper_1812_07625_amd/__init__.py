"""MI355X-native conv-GLU + CTC training path (wav2letter++ acoustic-model hot path).

The product is ``libw2l.so`` (hand-written HIP for gfx950 behind a C ABI, see
``include/w2l.h``); this package is the thin binding that marshals torch device
tensors into it.  There is no CPU fallback: the first use of any entry point loads the
library and raises if it has not been built (``python -m paper_1812_07625_amd.build``).
The binding is resolved lazily so that the build module can be imported before the
library exists.
"""
import importlib
import types

_binding = None
_found = {}  # entry points of the binding that this module holds as well by now


class _Binding(types.ModuleType):
    """The binding, which tells this module of entry points that are replaced in it (to trace them, in a test): they are looked up again."""

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        _forget(name)

    def __delattr__(self, name):
        super().__delattr__(name)
        _forget(name)


def _forget(name):
    for n in list(_found) if name.startswith("__") else [name]:  # (__spec__ and the like: the binding is loaded again)
        if n in _found and globals().get(n) is _found[n]:  # (not what a program has put in its place here)
            del globals()[n], _found[n]


def _load_binding():
    global _binding
    if _binding is None:
        _binding = importlib.import_module(".binding", __name__)
        _binding.__class__ = _Binding
    return _binding


def __getattr__(name):
    if name.startswith("__"):
        raise AttributeError(name)
    if name in ("build", "binding"):
        return importlib.import_module("." + name, __name__)
    value = getattr(_load_binding(), name)
    if callable(value) and not name.startswith("_"):
        globals()[name] = _found[name] = value  # found without this call from now on: 0.4 us of a call that takes 8
    return value


def __dir__():
    return sorted(set(globals()) | set(dir(_load_binding())))
