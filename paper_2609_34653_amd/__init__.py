"""OmniTide's per-chunk stream step on AMD Instinct MI355X (gfx950).

The product is ``libomnitide.so`` (hand-written HIP kernels behind the C ABI declared in
``include/omnitide.h``).  ``omnitide`` is its thin ctypes binding (same function names) and
``step.StreamStep`` drives one score -> select -> compact -> attend step on a HIP stream.  ``paged``
binds the calls of ``include/omnitide_paged.h``: a paged cache that streams of different lengths
share, what writes it and what reads it.
"""
from . import omnitide, paged  # noqa: F401
from .omnitide import OmnitideError, lib, version  # noqa: F401

__all__ = ["omnitide", "paged", "OmnitideError", "lib", "version"]
