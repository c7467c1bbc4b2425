"""Carry-through checksum CNN inference on MI355X (gfx950).

``ctc`` is the ctypes binding of libctc.so (include/ctc.h); ``CtcNet`` owns
a bound network; ``ops`` holds the operators around a protected classifier
(group norm, 8-bit products, token scores, attention over a map's pixels,
head norms with rotations, clipping of gradients).  Importing fails if the HIP
library is not built; ``ops`` is imported when it is first used, and fails
if its binding is not.
"""
from . import ctc  # noqa: F401
from .runtime import CtcNet  # noqa: F401


def __getattr__(name):
    if name == "ops":
        import importlib
        return importlib.import_module(".ops", __name__)
    raise AttributeError("module %r has no attribute %r" % (__name__, name))
