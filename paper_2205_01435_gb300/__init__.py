"""GB300-native world-model dream engine (RLFlow, SIGMOD'22): C ABI + thin binding.

The CUDA library ``libwm.so`` holds every kernel; ``wm`` marshals arguments.
Build it with ``__graft_entry__.build()`` (or ``python -m paper_2205_01435_gb300._build``).

``load()`` gives the world model's binding, ``load_seq()`` the sequence operators' (a gated
recurrent block's embedding, layer norm, scan over time and gradient clipping).
"""
from . import _build  # noqa: F401


def load():
    """Imports the ctypes binding; raises ImportError if libwm.so has not been built."""
    from . import wm
    return wm


def load_seq():
    """Imports the sequence operators' binding; raises ImportError if libwm.so or _seq_ext.so has not been built."""
    from . import seq
    return seq
