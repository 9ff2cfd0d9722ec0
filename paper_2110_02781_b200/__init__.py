"""B200-native per-stage training library (C ABI in include/ftpipe.h) and its thin Python binding.

The binding (and with it the shared library) is loaded on first use, so that
`python -m paper_2110_02781_b200.build` can run before the library exists or after its ABI changed.
"""
import importlib
import types

_copied = set()


class _Binding(types.ModuleType):
    """The binding's module.  The package keeps copies of the calls and constants asked for (0.4 us less a lookup); one that is
    replaced in the binding is forgotten here."""

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        _forget(name)

    def __delattr__(self, name):
        super().__delattr__(name)
        _forget(name)


def _forget(name):
    if name in _copied:
        _copied.discard(name)
        globals().pop(name, None)


def __getattr__(name):
    if name in ("build", "replicas"):                      # plain submodules: never need the library
        return importlib.import_module("." + name, __name__)
    ft = importlib.import_module(".ftpipe", __name__)      # raises if libftpipe.so is missing: there is no fallback
    ft.__class__ = _Binding
    try:
        value = getattr(ft, name)
    except AttributeError:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}") from None
    if not name.startswith("_") and (callable(value) or isinstance(value, int)):
        _copied.add(name)
        globals()[name] = value
    return value
