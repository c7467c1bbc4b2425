"""Carry-through checksum CNN inference on MI355X (gfx950).

``ctc`` is the ctypes binding of libctc.so (include/ctc.h); ``CtcNet`` owns
a bound network; ``ops`` holds the operators around a protected classifier
(group norm, 8-bit products, token scores).  Importing fails if the HIP library is not built.
"""
from . import ctc  # noqa: F401
from . import ops  # noqa: F401
from .runtime import CtcNet  # noqa: F401
