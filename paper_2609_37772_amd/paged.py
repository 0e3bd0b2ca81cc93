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
    """

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int,
                 max_seqs: int, dtype: torch.dtype = torch.bfloat16, rope_dim: int = 0, rope_theta: float = 10000.0,
                 rope_pairs: bool = False, k_scale: float = 1.0, v_scale: float = 1.0, device: int = 0,
                 stream: Optional[torch.cuda.Stream] = None, k: Optional[torch.Tensor] = None,
                 v: Optional[torch.Tensor] = None):
        self.handle = None
        if dtype not in _POOL_TYPES:
            raise ValueError(f"pools must be bfloat16 or float8_e4m3fn, got {dtype}")
        self.device = device
        self.n_layers, self.n_heads, self.n_kv_heads, self.head_dim = n_layers, n_heads, n_kv_heads, head_dim
        self._kv_row, self._q_row = (n_kv_heads, head_dim), (n_heads, head_dim)
        self._scale = 1.0 / math.sqrt(head_dim)
        shapes = ((n_layers, n_pages, n_kv_heads, page_size, head_dim), (n_layers, n_pages, n_kv_heads, head_dim, page_size))
        pools = []
        for name, pool, shape in zip("kv", (k, v), shapes):
            if pool is None:
                stream = stream or torch.cuda.current_stream(device)
                with torch.cuda.stream(stream):
                    pool = torch.empty(shape, dtype=dtype, device=torch.device("cuda", device))
            B._dev_ptr(pool, dtype, shape, name, device)
            pools.append(pool)
        self.k, self.v = pools
        self._stream = stream = stream or torch.cuda.current_stream(device)
        self._raw_stream = stream.cuda_stream
        self.handle = B.uad_kv_create(
            n_layers, n_heads, n_kv_heads, head_dim, page_size, n_pages, max_seqs, _POOL_TYPES[dtype], rope_dim,
            int(rope_pairs), rope_theta, k_scale, v_scale, self.k, self.v, device, stream)

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
            with torch.cuda.stream(self._stream):  # memory that another stream's queued work still uses is not taken
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            if _current_stream(self.device) != self._raw_stream:  # the caller's use of it as well
                out.record_stream(torch.cuda.current_stream(self.device))
        B.uad_kv_attend(self.handle, layer, q, out, page_table, lens, positions, self._scale if scale is None else scale,
                        self._q_row, self.device)
        if _current_stream(self.device) != self._raw_stream:
            self._used(q, out, page_table, lens, positions)
        return out

    def set_stream(self, stream: Optional[torch.cuda.Stream]) -> None:
        B.uad_kv_set_stream(self.handle, stream)
        self._stream = stream or torch.cuda.default_stream(self.device)
        self._raw_stream = self._stream.cuda_stream

    def synchronize(self) -> None:
        B.uad_kv_synchronize(self.handle)
