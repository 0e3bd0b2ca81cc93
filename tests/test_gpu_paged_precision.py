"""Attention is in fp32 and rounded once, for bf16 rows too: values that lie in the last third of an fp32 mantissa decide
the result here.  A value is split into bf16 parts (hi, then lo of what is left); what is left after two of them is what
the outputs are made of."""
import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
from tests.paged_oracle import U32
from tests.test_gpu_paged import BF16, F32, dev

HD, PAGE = 64, 16


def parts(x):
    """hi, lo (bf16 values) and what is left of x, in 64 bits."""
    hi = torch.tensor(x, dtype=torch.float64).to(BF16).double().numpy()
    lo = torch.tensor(x - hi, dtype=torch.float64).to(BF16).double().numpy()
    return hi, lo, x - hi - lo


def cache(seqs, tokens, heads, rope):
    """A cache of one page per sequence, and its keys and values by [sequence][token][dim] for the caller to fill."""
    kv = U.PagedKV(1, heads, 1, HD, PAGE, seqs, seqs, rope_dim=rope)
    kv.k.zero_(), kv.v.zero_()
    return kv, kv.k[0, :, 0, :tokens], kv.v[0, :, 0, :, :tokens].transpose(1, 2), torch.arange(seqs, dtype=torch.int32, device="cuda")[:, None].contiguous()


def weights_case():
    """Scores 0, 0 and -c: weights 1, 1 and w = e^-c; values -hi, -lo and 1, so that the sum is what is left of w."""
    c = torch.arange(0.25, 4.0, 2.0 ** -7).to(BF16).double().unique().numpy()
    w = np.exp(-c)
    hi, lo, rest = parts(w)
    # the sum: w off by its exponential (2^-21) and its score (two roundings of c), and three roundings at up to 2 w; the
    # denominator's error counts for nothing beside that
    off = w * (2.0 ** -21 + 2 * U32 * c + 6 * U32) / (2 + w)
    best = np.argsort(-np.abs(rest) / w)[:24]
    c, w, hi, lo, rest, off = (x[best] for x in (c, w, hi, lo, rest, off))
    return c, hi, lo, rest / (2 + w), off


def test_the_weights_case_tells_two_parts_from_three():
    _, _, _, out, off = weights_case()
    assert np.all(np.abs(out) > 2 * off)  # with w = hi + lo the sum is 0


def query_case():
    """A query (1, 0) turned by a position: cos of it, times 256, against a key that holds hi and lo of that where the
    query is 1 and not turned.  Values 1 and -1: the output is tanh of half of what is left."""
    positions = np.arange(1, 4000)
    x = 256 * np.cos(positions.astype(np.float64))
    hi, lo, rest = parts(x)
    best = np.argsort(-np.abs(rest) * (np.abs(x) > 128))[:24]
    out = np.tanh(rest[best] / 2)
    # scores: 16 u of 256 for the turn, three terms of up to 512; half of their difference, and the exponential's 2^-21
    off = (256 * 16 * U32 + 6 * 512 * U32) / 2 + 2 * 2.0 ** -21
    return positions[best], hi[best], lo[best], out, off


def test_the_query_case_tells_two_parts_from_three():
    _, _, _, out, off = query_case()
    assert np.all(np.abs(out) > 2 * off)


@pytest.mark.gpu
@pytest.mark.parametrize("given", [BF16, F32])
def test_weights_keep_what_fp32_holds(gpu, given):
    c, hi, lo, want, off = weights_case()
    n = len(c)
    kv, k, v, table = cache(n, 3, 1, 0)
    k[:, 2, 0] = dev(-c).to(BF16)
    v[:, 0], v[:, 1], v[:, 2] = dev(-hi)[:, None].to(BF16), dev(-lo)[:, None].to(BF16), 1.0
    q = torch.zeros((n, 1, HD), dtype=given, device="cuda")
    q[..., 0] = 1.0
    got = kv.attend(0, q, table, torch.full((n,), 3, dtype=torch.int32, device="cuda"), scale=1.0)
    kv.synchronize()
    off = off + np.abs(want) * 2.0 ** (-8 if given == BF16 else -24)
    assert np.all(np.abs(got[:, 0].double().cpu().numpy() - want[:, None]) <= off[:, None])


@pytest.mark.gpu
@pytest.mark.parametrize("given", [BF16, F32])
def test_turned_queries_keep_what_fp32_holds(gpu, given):
    positions, hi, lo, want, off = query_case()
    n = len(positions)
    kv, k, v, table = cache(n, 2, 1, 16)
    k[:, 0, 0] = 256.0
    k[:, 1, 40], k[:, 1, 41] = dev(hi).to(BF16), dev(lo).to(BF16)
    v[:, 0], v[:, 1] = 1.0, -1.0
    q = torch.zeros((n, 1, HD), dtype=given, device="cuda")
    q[..., 0] = q[..., 40] = q[..., 41] = 1.0
    got = kv.attend(0, q, table, torch.full((n,), 2, dtype=torch.int32, device="cuda"), positions=dev(positions.astype(np.int32)), scale=1.0)
    kv.synchronize()
    off = off + np.abs(want) * 2.0 ** (-8 if given == BF16 else -24)
    assert np.all(np.abs(got[:, 0].double().cpu().numpy() - want[:, None]) <= off[:, None])
