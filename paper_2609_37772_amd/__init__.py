"""Urgency-Aware Denoising (UAD) action-expert hot path for AMD MI355X (gfx950).

The compute runs in ``libuad.so`` (hand-written HIP kernels behind the C ABI
of ``include/uad.h``); this package is its thin Python binding plus a small
convenience wrapper, :class:`ActionExpert`, used by the tests and the benchmark,
and :class:`PagedKV`, the paged K/V cache that an expert can take its prefix from.
"""
from ._binding import *  # noqa: F401,F403
from ._binding import __all__ as _b_all
from .expert import ActionExpert
from .paged import PagedKV

__all__ = list(_b_all) + ["ActionExpert", "PagedKV"]
