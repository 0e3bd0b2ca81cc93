"""Convenience wrapper owning one paged K/V cache: its pools and its libuad handle (marshalling only)."""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import _binding as B

_current_stream = torch._C._cuda_getCurrentRawStream  # of a device, as its handle
_POOL_TYPES = {torch.bfloat16: B.UAD_DTYPE_BF16, torch.float8_e4m3fn: B.UAD_DTYPE_F8}


class PagedKV:
    """The paged K/V cache of a vision-language model on one GPU (see the uad_kv entry points in include/uad.h).

    ``k`` [n_layers][n_pages][n_kv_heads][page_size][head_dim] and ``v`` (pages transposed:
    [n_layers][n_pages][n_kv_heads][head_dim][page_size]) are allocated when not given.  Work goes to ``stream`` (the
    current one when not given), which tensors that a call allocates belong to, whichever stream is current: what a call
    reads has to be there by the time that ``stream`` gets to it, and must not change until it has.  Called from another
    stream, it keeps its tensors' memory from being reused before that.

    ``block_scales``: float8_e4m3fn pools with a scale of their own for every 16 tokens and KV head, which ``append``
    finds (see uad_kv_set_block_scales); ``k_scales`` and ``v_scales`` [n_layers][n_pages][n_kv_heads][page_size // 16] are
    allocated when not given.
    """

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int,
                 max_seqs: int, dtype: torch.dtype = torch.bfloat16, rope_dim: int = 0, rope_theta: float = 10000.0,
                 rope_pairs: bool = False, k_scale: float = 1.0, v_scale: float = 1.0, device: int = 0,
                 stream: Optional[torch.cuda.Stream] = None, k: Optional[torch.Tensor] = None,
                 v: Optional[torch.Tensor] = None, block_scales: bool = False, k_scales: Optional[torch.Tensor] = None,
                 v_scales: Optional[torch.Tensor] = None):
        self.handle = None
        if dtype not in _POOL_TYPES:
            raise ValueError(f"pools must be bfloat16 or float8_e4m3fn, got {dtype}")
        if block_scales and (dtype != torch.float8_e4m3fn or k_scale != 1.0 or v_scale != 1.0):
            raise ValueError("block_scales are for float8_e4m3fn pools with k_scale and v_scale 1")
        if not block_scales and (k_scales is not None or v_scales is not None):
            raise ValueError("k_scales and v_scales need block_scales")
        self.device = device
        self.n_pages = n_pages
        self.n_layers, self.n_heads, self.n_kv_heads, self.head_dim = n_layers, n_heads, n_kv_heads, head_dim
        self._kv_row, self._q_row = (n_kv_heads, head_dim), (n_heads, head_dim)
        self._scale = 1.0 / math.sqrt(head_dim)
        shapes = ((n_layers, n_pages, n_kv_heads, page_size, head_dim), (n_layers, n_pages, n_kv_heads, head_dim, page_size))

        def owned(name, given, dtype, shape):
            nonlocal stream
            if given is None:
                stream = stream or torch.cuda.current_stream(device)
                with torch.cuda.stream(stream):
                    given = torch.empty(shape, dtype=dtype, device=torch.device("cuda", device))
            B._dev_ptr(given, dtype, shape, name, device)
            return given

        self.k, self.v = (owned(n, t, dtype, shape) for n, t, shape in zip("kv", (k, v), shapes))
        self.k_scales = self.v_scales = None
        if block_scales:
            shape = (n_layers, n_pages, n_kv_heads, page_size // 16)
            self.k_scales, self.v_scales = (owned(n, t, torch.float32, shape)
                                            for n, t in (("k_scales", k_scales), ("v_scales", v_scales)))
        self._stream = stream = stream or torch.cuda.current_stream(device)
        self._raw_stream = stream.cuda_stream
        self.handle = B.uad_kv_create(
            n_layers, n_heads, n_kv_heads, head_dim, page_size, n_pages, max_seqs, _POOL_TYPES[dtype], rope_dim,
            int(rope_pairs), rope_theta, k_scale, v_scale, self.k, self.v, device, stream)
        if block_scales:
            B.uad_kv_set_block_scales(self.handle, self.k_scales, self.v_scales)

    def close(self):
        if getattr(self, "handle", None):
            B.uad_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _used(self, *tensors) -> None:
        """The memory of tensors that another stream's call brought is in use on the handle's."""
        for t in tensors:
            if t is not None:
                t.record_stream(self._stream)

    def append(self, layer: int, k, v, page_table, lens, row_start=None, positions=None) -> None:
        """Append new tokens' keys (rotated) and values to a layer; see uad_kv_append."""
        B.uad_kv_append(self.handle, layer, k, v, page_table, lens, row_start, positions, self._kv_row, self.device)
        if _current_stream(self.device) != self._raw_stream:
            self._used(k, v, page_table, lens, row_start, positions)

    def attend(self, layer: int, q, page_table, lens, out=None, positions=None, scale: Optional[float] = None):
        """Attention of one token per sequence; see uad_kv_attend.  Allocates ``out`` when not given and returns it."""
        if out is None:
            out = self._like(q)
        B.uad_kv_attend(self.handle, layer, q, out, page_table, lens, positions, self._scale if scale is None else scale,
                        self._q_row, self.device)
        if _current_stream(self.device) != self._raw_stream:
            self._used(q, out, page_table, lens, positions)
        return out

    def _like(self, q) -> torch.Tensor:
        with torch.cuda.stream(self._stream):  # memory that another stream's queued work still uses is not taken
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if _current_stream(self.device) != self._raw_stream:  # the caller's use of it as well
            out.record_stream(torch.cuda.current_stream(self.device))
        return out

    def attend_rows(self, layer: int, q, page_table, lens, row_start=None, out=None, positions=None,
                    scale: Optional[float] = None, window: int = 0, sinks: int = 0, causal: bool = True):
        """Attention of the newest rows of every sequence, or of one each without ``row_start``, with a sliding window
        and sinks; see uad_kv_attend_rows.  Allocates ``out`` when not given and returns it."""
        if out is None:
            out = self._like(q)
        B.uad_kv_attend_rows(self.handle, layer, q, out, page_table, lens, row_start, positions,
                             self._scale if scale is None else scale, window, sinks, causal, self._q_row, self.device)
        if _current_stream(self.device) != self._raw_stream:
            self._used(q, out, page_table, lens, row_start, positions)
        return out

    def reserve(self, lens, page_table, free_pages, n_free, new_tokens=None, row_start=None, slots=None, lens_out=None,
                n_free_out=None) -> None:
        """Take the pages of new tokens (one for each sequence without ``new_tokens``) from the free ones; see uad_kv_reserve.
        ``lens`` and ``n_free`` are updated in place, or go to ``lens_out`` and ``n_free_out`` where given."""
        lens_out, n_free_out = lens if lens_out is None else lens_out, n_free if n_free_out is None else n_free_out
        B.uad_kv_reserve(self.handle, lens, page_table, free_pages, n_free, new_tokens, row_start, slots, lens_out, n_free_out,
                         self.n_pages, self.device)
        if _current_stream(self.device) != self._raw_stream:
            self._used(lens, page_table, free_pages, n_free, new_tokens, row_start, slots, lens_out, n_free_out)

    def release(self, lens, page_table, free_pages, n_free, window: int = 0, sinks: int = 0) -> None:
        """Give back the pages that no later token sees; see uad_kv_release."""
        B.uad_kv_release(self.handle, lens, page_table, free_pages, n_free, window, sinks, self.n_pages, self.device)
        if _current_stream(self.device) != self._raw_stream:
            self._used(lens, page_table, free_pages, n_free)

    def set_stream(self, stream: Optional[torch.cuda.Stream]) -> None:
        B.uad_kv_set_stream(self.handle, stream)
        self._stream = stream or torch.cuda.default_stream(self.device)
        self._raw_stream = self._stream.cuda_stream

    def synchronize(self) -> None:
        B.uad_kv_synchronize(self.handle)
