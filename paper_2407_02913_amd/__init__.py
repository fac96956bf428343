"""SFC (Symbolic Fourier Convolution) 3x3 int8 convolution for MI355X (gfx950).

The compute path is a C-ABI shared library of hand-written HIP kernels
(``csrc/``, declared in ``include/sfc.h``); :mod:`.binding` marshals arguments
to it and nothing else.  There is no CPU fallback: calling into the library
when it has not been built raises.  :mod:`.adapt` holds the operators around the
convolutions: what is tuned and served beside their frozen weights.
"""
from . import synth  # noqa: F401

__all__ = ["synth", "binding", "adapt"]


def __getattr__(name):
    if name in ("binding", "adapt"):
        import importlib

        return importlib.import_module("." + name, __name__)
    raise AttributeError(name)
