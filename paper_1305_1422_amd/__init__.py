"""Batch self-organizing-map training on one AMD MI355X: binding of the HIP library libsom.

``capi`` mirrors ``include/som.h`` name for name; ``Som`` is a convenience wrapper holding
torch tensors, ``Mx4`` rows in microscaled 4-bit form.  The library must have been built (``python -m paper_1305_1422_amd.build``).
"""
from . import capi  # noqa: F401

__all__ = ["capi", "Mx4", "Som"]


def __getattr__(name):
    if name in ("Som", "Mx4"):
        from . import som
        return getattr(som, name)
    raise AttributeError(name)
