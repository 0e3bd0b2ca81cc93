"""Attention of new rows, appends with scales for blocks and page tables, from their definitions in 64 bits and in plain
Python, and how far fp32 kernels may be off (see paged_oracle)."""
from __future__ import annotations

import numpy as np
import torch

from tests import paged_oracle as P
from tests.paged_oracle import U32

F8 = torch.float8_e4m3fn
BLOCK = 16


class Cache(P.Cache):
    """paged_oracle's cache, in 8 bits with a scale for every block of 16 tokens and KV head where `blocks`."""

    def __init__(self, seed, layers, hkv, hd, page, lens, blocks=False, cache=torch.bfloat16, poison=float("nan"), **kw):
        super().__init__(seed, layers, hkv, hd, page, lens, cache=F8 if blocks else cache, poison=poison, **kw)
        self.blocks = blocks
        if blocks:
            self.scales = (1.0, 1.0)
            shape = (layers, self.n_pages, hkv, page // BLOCK)
            self.block = [torch.full(shape, poison) for _ in range(2)]

    def fill(self, seed, layer=None, spread=1.0):
        if not self.blocks:
            return super().fill(seed, layer, spread)
        g = torch.Generator().manual_seed(seed)
        for l in range(self.layers) if layer is None else [layer]:
            for b, n in enumerate(self.lens):
                for at in range(0, int(n), BLOCK):
                    p, off = self.slot(b, at)
                    m = min(BLOCK, int(n) - at)
                    # scales that are no powers of two too: the caller may have any
                    ks, vs = (2.0 ** torch.randint(-8, -5, (2, self.hkv), generator=g) * (1 + 0.25 * torch.rand(2, self.hkv, generator=g)))
                    self.block[0][l, p, :, off // BLOCK], self.block[1][l, p, :, off // BLOCK] = ks, vs
                    self.k[l, p, :, off:off + m] = (100 * spread * torch.randn(self.hkv, m, self.hd, generator=g)).clamp(-448, 448).to(F8)
                    self.v[l, p, :, :, off:off + m] = (100 * torch.randn(self.hkv, self.hd, m, generator=g)).clamp(-448, 448).to(F8)

    def tokens(self, layer, b, n=None):
        k, v = super().tokens(layer, b, n)
        if self.blocks:
            at = np.arange(len(k))
            page, sub = self.table[b, at // self.page], at % self.page // BLOCK
            k, v = (x * s[layer].double().numpy()[page, :, sub][..., None] for x, s in zip((k, v), self.block))
        return k, v

    def hide(self, new, window, sinks):
        """Page table entries that no row sees become -9, and what lies in such pages NaN."""
        if not window:
            return
        for b, (n, m) in enumerate(zip(new, self.lens)):
            for i in range(-(-int(m) // self.page)):
                x = np.arange(i * self.page, min((i + 1) * self.page, int(m)))
                if not np.any((x < sinks) | (x > int(m) - n - window)):
                    self.table[b, i] = -9


def sees(n, m, window, sinks, causal):
    """[n][m] whether the rows of the last n of m tokens see the keys."""
    p, x = np.arange(m - n, m)[:, None], np.arange(m)[None]
    mask = x <= p if causal else np.ones((n, m), bool)
    if window:
        mask = mask & ((np.abs(p - x) < window) | (x < sinks))
    return mask


def attend_rows(cache, layer, q, new, rope, pairs, scale, window=0, sinks=0, causal=True, positions=None, theta=10000.0):
    """Exact outputs [rows][heads][hd], sum p |v|, the largest sum |q k| * |scale| of each (row, head) over the keys that it
    sees, and the number of those."""
    q = np.asarray(q, np.float64)
    rows, heads, hd = q.shape
    o, b_, a_, n_ = np.zeros(q.shape), np.zeros(q.shape), np.zeros((rows, heads, 1)), np.zeros((rows, 1, 1))
    at = 0
    for b, n in enumerate(new):
        m = int(cache.lens[b])
        if n == 0 or m == 0:
            at += n
            continue
        mask = sees(n, m, window, sinks, causal)
        x = np.flatnonzero(mask.any(0))  # tokens that a row sees; the others may lie in no page
        mask = mask[:, x]
        old = cache.table[b].copy()
        cache.table[b] = np.maximum(cache.table[b], 0)
        k, v = (t[x] for t in cache.tokens(layer, b))
        cache.table[b] = old
        turn = np.arange(m - n, m) if positions is None else np.asarray(positions[at:at + n])
        r, _ = P.rotate(q[at:at + n], turn, rope, pairs, theta)
        n_[at:at + n, 0, 0] = mask.sum(1)
        for h in range(heads):
            g = h * cache.hkv // heads
            s = np.where(mask, scale * (r[:, h] @ k[:, g].T), -np.inf)
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            o[at:at + n, h], b_[at:at + n, h] = w @ v[:, g], w @ np.abs(v[:, g])
            a_[at:at + n, h, 0] = np.where(mask, abs(scale) * (np.abs(r[:, h]) @ np.abs(k[:, g]).T), 0).max(1)
        at += n
    return o, b_, a_, n_


def rows_bound(o, b, n, hd, a, terms, dtype):
    """As paged_oracle's attend_bound, queries and weights in `terms` bf16 parts, with a block's scale on the score and on the
    weight (a rounding each)."""
    ds = a * ((hd + 26) * U32 + 2.0 ** (-8 * terms))
    rel = 2 * (ds * 1.5 + 2.0 ** -21 + 2.0 ** (-8 * terms)) + 2 * (n + 18) * U32
    off = rel * b
    return off + P.half_step(np.abs(o) + off, dtype)


def block_scale(most):
    """The least power of two from 2^-100 to 2^119 by which `most` is within 448."""
    e = -100
    while e < 119 and 448.0 * 2.0 ** e < most:
        e += 1
    return 2.0 ** e


class Pages:
    """The page tables' calls in plain Python."""

    def __init__(self, page, n_pages, table, lens, free):
        self.page, self.n_pages = page, n_pages
        self.table, self.lens, self.free = [list(map(int, r)) for r in table], [int(x) for x in lens], [int(x) for x in free]

    def reserve(self, new):
        """(row starts, slots), or None where nothing is taken."""
        p = self.page
        need = [-(-(m + n) // p) - -(-m // p) for m, n in zip(self.lens, new)]
        if sum(need) > len(self.free) or any(m + n > len(r) * p for m, n, r in zip(self.lens, new, self.table)):
            return None
        starts, slots = [0], []
        for b, n in enumerate(new):
            for x in range(self.lens[b], self.lens[b] + n):
                if x % p == 0:
                    self.table[b][x // p] = self.free.pop()
                slots.append(self.table[b][x // p] * p + x % p)
            self.lens[b] += n
            starts.append(starts[-1] + n)
        return starts, slots

    def release(self, window, sinks):
        for b, m in enumerate(self.lens):
            for i, id in enumerate(self.table[b]):
                kept = any(x < sinks or window == 0 or x > m - window for x in range(i * self.page, min(m, (i + 1) * self.page)))
                kept = kept or (m % self.page > 0 and i == m // self.page)
                if id >= 0 and not kept:
                    self.free.append(id)
                    self.table[b][i] = -1
