"""zkmi: the tlookup / sumcheck prover hot path of zkLLM on one AMD MI355X.

The work is done by ``libzkmi.so`` (hand-written HIP for gfx950, built in-tree by
``paper_2404_16109_amd.build``); this package is argument marshalling only.
PyTorch is used to own device memory and to name the stream.  There is no CPU
fallback: the first use of any entry point loads the library and raises if it
has not been built.  (``paper_2404_16109_amd.build`` and ``.synth`` can be
imported without it.)
"""
import importlib
import types


_kept = set()  # the binding's names that the package has found and holds


class _Binding(types.ModuleType):
    """The binding: a name that is set or deleted in it later is looked up anew by the package."""

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        _forget(name)

    def __delattr__(self, name):
        super().__delattr__(name)
        _forget(name)


def _forget(name):
    if name in _kept:
        _kept.discard(name)
        globals().pop(name, None)


def __getattr__(name):
    if name.startswith("__"):
        raise AttributeError(name)
    if name in ("build", "synth", "binding"):
        return importlib.import_module("." + name, __name__)
    binding = importlib.import_module(".binding", __name__)
    binding.__class__ = _Binding
    value = getattr(binding, name)
    _kept.add(name)
    globals()[name] = value  # found without this detour from now on: it costs as much as a launch
    return value
