"""Attention of new rows is in fp32 and rounded once, whichever kernel the size of a call picks: the cases of
test_gpu_paged_precision, whose outputs are made of what two bf16 parts leave out, with sequences of 16 rows that all see
the same few keys, in calls large enough for the kernel of many rows."""
import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
from tests.paged_oracle import U32
from tests.test_gpu_paged import BF16, F32, dev
from tests.test_gpu_paged_precision import parts, query_case

ROWS, GROUP = 16, 32
# head dim, KV heads: two waves a column, and one
SIZES = [(hd, hkv) for hd in (64, 128, 256) for hkv in (1, 3)]


def weights_case():
    """As there, with smaller c and this kernel's roundings: scores of -c are off by the one of log2(e) and up to four of
    sums, weights by their exponential (2^-21), and three sums are rounded at up to 2 w."""
    c = np.arange(0.25, 1.0, 2.0 ** -7)
    w = np.exp(-c)
    hi, lo, rest = parts(w)
    off = w * (2.0 ** -21 + 5 * U32 * c + 6 * U32) / (2 + w)
    best = np.argsort(-np.abs(rest) / w)[:24]
    c, w, hi, lo, rest, off = (x[best] for x in (c, w, hi, lo, rest, off))
    return c, hi, lo, rest / (2 + w), off


def turned_case():
    """As there; queries are scaled before they are split into parts, which rounds the turned one once more, at up to 256
    times its key (the others are 1)."""
    positions, hi, lo, want, off = query_case()
    return positions, hi, lo, want, off + 256 * U32 / 2


def test_the_cases_tell_two_parts_from_three():
    for _, _, _, out, off in (weights_case(), turned_case()):
        assert np.all(np.abs(out) > 2 * off)


def cache(seqs, hd, hkv, rope):
    """A page of 16 tokens a sequence; keys and values by [sequence][KV head][token][dim] for the caller to fill."""
    kv = U.PagedKV(1, hkv * GROUP, hkv, hd, 16, seqs, seqs, rope_dim=rope)
    kv.k.zero_(), kv.v.zero_()
    ints = lambda *a: torch.arange(*a, dtype=torch.int32, device="cuda")  # noqa: E731
    lens = torch.full((seqs,), 16, dtype=torch.int32, device="cuda")
    return kv, kv.k[0], kv.v[0].transpose(2, 3), ints(seqs)[:, None].contiguous(), lens, ints(0, ROWS * seqs + 1, ROWS)


def check(got, want, off, given):
    off = off + np.abs(want) * 2.0 ** (-8 if given == BF16 else -22)
    got = got.double().cpu().numpy().reshape(len(want), -1)
    assert np.all(np.abs(got - want[:, None]) <= off[:, None]), float((np.abs(got - want[:, None]) / off[:, None]).max())


@pytest.mark.gpu
@pytest.mark.parametrize("hd,hkv", SIZES)
@pytest.mark.parametrize("given", [BF16, F32])
def test_weights_keep_what_fp32_holds(gpu, given, hd, hkv):
    c, hi, lo, want, off = weights_case()
    n = len(c)
    kv, k, v, table, lens, starts = cache(n, hd, hkv, 0)
    k[:, :, 3:, 0] = -1024.0  # of no weight
    k[:, :, 2, 0] = dev(-c).to(BF16)[:, None]
    v[:, :, 0], v[:, :, 1], v[:, :, 2] = dev(-hi).to(BF16)[:, None, None], dev(-lo).to(BF16)[:, None, None], 1.0
    q = torch.zeros((n * ROWS, hkv * GROUP, hd), dtype=given, device="cuda")
    q[..., 0] = 1.0
    got = kv.attend_rows(0, q, table, lens, starts, scale=1.0, causal=False)
    kv.synchronize()
    check(got, want, off, given)


@pytest.mark.gpu
@pytest.mark.parametrize("hd,hkv", SIZES)
@pytest.mark.parametrize("given", [BF16, F32])
def test_turned_queries_keep_what_fp32_holds(gpu, given, hd, hkv):
    positions, hi, lo, want, off = turned_case()
    n = len(positions)
    kv, k, v, table, lens, starts = cache(n, hd, hkv, 16)
    k[:, :, 2:, 50] = -4096.0  # of no weight
    k[:, :, 0, 0] = 256.0
    k[:, :, 1, 40], k[:, :, 1, 41] = dev(hi).to(BF16)[:, None], dev(lo).to(BF16)[:, None]
    v[:, :, 0], v[:, :, 1] = 1.0, -1.0
    q = torch.zeros((n * ROWS, hkv * GROUP, hd), dtype=given, device="cuda")
    q[..., 0] = q[..., 40] = q[..., 41] = q[..., 50] = 1.0
    at = dev(np.repeat(positions, ROWS).astype(np.int32))
    got = kv.attend_rows(0, q, table, lens, starts, positions=at, scale=1.0, causal=False)
    kv.synchronize()
    check(got, want, off, given)
