"""OmniTide's per-chunk stream step on AMD Instinct MI355X (gfx950).

The product is ``libomnitide.so`` (hand-written HIP kernels behind the C ABI declared in
``include/omnitide.h``).  ``omnitide`` is its thin ctypes binding (same function names) and
``step.StreamStep`` drives one score -> select -> compact -> attend step on a HIP stream.  ``paged``
binds the calls of ``include/omnitide_paged.h``: a paged cache that streams of different lengths
share, what writes it and what reads it; ``latent`` those of ``include/omnitide_latent.h``, a paged cache
of latent vectors, and ``evict`` those of ``include/omnitide_evict.h``: eviction by attention weight.
"""
from . import evict, latent, omnitide, paged  # noqa: F401
from .omnitide import OmnitideError, lib, version  # noqa: F401

__all__ = ["evict", "latent", "omnitide", "paged", "OmnitideError", "lib", "version"]
