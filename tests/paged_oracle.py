"""The paged cache's operators in 64 bits, token by token from their definitions, and how far fp32 kernels may be off.

Bounds are sums of what each step may lose: a rounding to a type is off by half a step at most (u = 2^-24 for fp32), a
dot product of n terms by n u times the sum of their magnitudes.
"""
from __future__ import annotations

import numpy as np
import torch

U32 = 2.0 ** -24


def rotation(positions, rope_dim, theta=10000.0):
    """cos, sin [positions][rope_dim / 2] in 64 bits."""
    i = np.arange(rope_dim // 2, dtype=np.float64)
    angle = np.asarray(positions, np.float64)[:, None] * theta ** (-2.0 * i / max(rope_dim, 1))
    return np.cos(angle), np.sin(angle)


def rotate(x, positions, rope_dim, pairs, theta=10000.0):
    """x [rows][heads][hd] turned by positions; also sum |a| + |b| of each element's pair (0 where nothing is turned)."""
    x = np.asarray(x, np.float64)
    out, size = x.copy(), np.zeros_like(x)
    cos, sin = rotation(positions, rope_dim, theta)
    for i in range(rope_dim // 2):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rope_dim // 2)
        c, s = cos[:, None, i], sin[:, None, i]
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return out, size


def half_step(x, dtype):
    """Half a step of `dtype` at magnitudes |x|."""
    x = np.abs(x)
    if dtype == torch.float8_e4m3fn:  # normal from 2^-6, steps of 2^-9 below
        return np.maximum(x * 2.0 ** -4, 2.0 ** -10)
    return x * {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}[dtype]


def append_bound(exact, size, scale, dtype):
    """Stored values: angle and products of the rotation in fp32 (the fraction of a turn rounded once: 2 pi u of angle;
    sine and cosine within 4 u; three roundings: under 16 u in all), 1/scale and the product with it (2 u), one rounding."""
    off = (16 * U32 * size + 2 * U32 * np.abs(exact)) / scale
    return off + half_step(np.abs(exact) / scale + off, dtype)


def attend_bound(o, b, n, hd, a, terms_q, terms_p, dtype):
    """o: exact output, b: sum p |v| of it, n: keys, a: the largest sum |q k| * scale over the keys.
    A score is off by (hd + 24) u a (dot product, rotation, scale) and what is left of q after terms_q bf16 terms; a
    weight by e^that, 2^-21 of its exponential and what is left of it after terms_p terms; numerator and denominator
    add n terms each."""
    ds = a * ((hd + 24) * U32 + 2.0 ** (-8 * terms_q))
    rel = 2 * (ds * 1.5 + 2.0 ** -21 + 2.0 ** (-8 * terms_p)) + 2 * (n + 16) * U32
    off = rel * b
    return off + half_step(np.abs(o) + off, dtype)


class Cache:
    """Pools with poison in every slot, shuffled pages, and a token-by-token copy of what they should hold."""

    def __init__(self, seed, layers, hkv, hd, page, lens, wide=None, cache=torch.bfloat16, spare=3, shared=None,
                 poison=float("nan")):
        g = np.random.default_rng(seed)
        self.hkv, self.hd, self.page, self.layers, self.dtype = hkv, hd, page, layers, cache
        self.scales = (0.03, 0.05) if cache == torch.float8_e4m3fn else (1.0, 1.0)
        need = [-(-n // page) for n in lens]
        wide = max(need + [1]) + 1 if wide is None else wide
        self.n_pages = sum(need) + spare
        ids = g.permutation(self.n_pages)
        self.table = np.full((len(lens), wide), -7, np.int32)
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = ids[at:at + m]
            at += m
        if shared:  # (from, to): whole pages of one sequence read by another
            self.table[shared[1], :shared[2]] = self.table[shared[0], :shared[2]]
        self.lens = np.asarray(lens, np.int32)
        self.k = torch.full((layers, self.n_pages, hkv, page, hd), poison, dtype=torch.float32).to(cache)
        self.v = torch.full((layers, self.n_pages, hkv, hd, page), poison, dtype=torch.float32).to(cache)

    def slot(self, b, pos):
        return int(self.table[b, pos // self.page]), pos % self.page

    def fill(self, seed, layer=None, spread=1.0):
        """Random tokens in every slot that the sequences hold."""
        g = torch.Generator().manual_seed(seed)
        for l in range(self.layers) if layer is None else [layer]:
            for b, n in enumerate(self.lens):
                for pg in range(-(-int(n) // self.page)):
                    m = min(self.page, int(n) - pg * self.page)
                    p = int(self.table[b, pg])
                    k = torch.randn((self.hkv, m, self.hd), generator=g) * spread
                    v = torch.randn((self.hkv, self.hd, m), generator=g)
                    self.k[l, p, :, :m] = (k / self.scales[0]).clamp(-448, 448).to(self.dtype)
                    self.v[l, p, :, :, :m] = (v / self.scales[1]).clamp(-448, 448).to(self.dtype)

    def tokens(self, layer, b, n=None):
        """K and V [tokens][hkv][hd] in 64 bits."""
        n = int(self.lens[b]) if n is None else n
        ids = torch.from_numpy(self.table[b, :-(-n // self.page)].astype(np.int64))
        k = self.k[layer].float()[ids].transpose(1, 2).reshape(-1, self.hkv, self.hd)[:n].double().numpy()
        v = self.v[layer].float()[ids].permute(0, 3, 1, 2).reshape(-1, self.hkv, self.hd)[:n].double().numpy()
        return k * self.scales[0], v * self.scales[1]


def attend(cache, layer, q, positions, rope_dim, pairs, scale, theta=10000.0):
    """Exact outputs [seqs][heads][hd], sum p |v|, and the largest sum |q k| * |scale| of each (seq, head)."""
    q, _ = rotate(q, positions, rope_dim, pairs, theta)
    seqs, heads, hd = q.shape
    o, b_, a_ = np.zeros(q.shape), np.zeros(q.shape), np.zeros((seqs, heads, 1))
    for b in range(seqs):
        if cache.lens[b] == 0:
            continue
        k, v = cache.tokens(layer, b)
        for h in range(heads):
            g = h * cache.hkv // heads
            s = scale * (k[:, g] @ q[b, h])
            w = np.exp(s - s.max())
            w /= w.sum()
            o[b, h], b_[b, h] = w @ v[:, g], w @ np.abs(v[:, g])
            a_[b, h, 0] = abs(scale) * (np.abs(k[:, g]) @ np.abs(q[b, h])).max()
    return o, b_, a_
