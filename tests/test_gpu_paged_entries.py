"""Lengths and starts that cannot be used, on the GPU: reported by whichever kernel an append takes, for every sequence,
and nothing is written on their account."""
import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
from tests import paged_oracle as P
from tests.test_gpu_paged import check_attend, dev, draw, handle

pytestmark = pytest.mark.gpu
WIDE, PAGE = 40, 16  # a table of 640 tokens

# sequences behind a first one with `most` rows: where their rows end (from there), their lengths, the rows that there
# are, and which of them are refused
BAD = {
    "rows that do not exist": ([3, 5], [3, 2], 3, [1]),
    "and a fall behind them": ([3, 5, 4], [3, 2, 0], 3, [1, 2]),
    "falls that leave each row a sequence": ([2, 1, 2, 2, 1], [40] * 5, 2, [1, 4]),
    "length below zero without rows": ([0, 2], [-1, 2], 2, [0]),
    "length beyond the table without rows": ([2, 2], [2, 641], 2, [1]),
    "length beyond the table": ([2, 4], [2, 641], 4, [1]),
    "length beyond any table": ([2, 4], [2 ** 31 - 1, 2], 4, [0]),
    "length below the rows": ([5, 6], [4, 1], 6, [0]),
}


@pytest.mark.parametrize("what", BAD)
@pytest.mark.parametrize("most", [1, 640], ids=["row by row", "by tiles"])
@pytest.mark.parametrize("others", [0, 70])  # sequences without rows or tokens, for more than a wave has lanes
def test_append_reports_and_writes_nothing(gpu, what, most, others):
    ends, lens, extra, refused = BAD[what]
    n, rows = 1 + len(ends) + others, most + extra
    assert (8 * n <= rows) == (most > 1)
    starts = np.array([0, most] + [most + x for x in ends] + [most + ends[-1]] * others, np.int32)
    lens = np.array([most, *lens] + [0] * others, np.int32)
    c = P.Cache(3, 1, 2, 64, PAGE, [most] + [48] * len(ends) + [0] * others, wide=WIDE, poison=0.5)
    spare = sorted(set(range(c.n_pages)) - set(c.table[c.table >= 0].tolist()))
    table = np.where(c.table < 0, spare[0], c.table).astype(np.int32)  # every entry is a page
    kv = handle(c, 2)
    k = dev(draw(1, rows, 2, 64))
    kv.append(0, k, k, dev(table), dev(lens), dev(starts))
    with pytest.raises(U.UadError) as e:
        kv.synchronize()
    assert e.value.status == 9
    kept = spare + [int(p) for b in refused for p in table[1 + b, :3]]
    assert bool((kv.k[0, kept] == 0.5).all()) and bool((kv.v[0, kept] == 0.5).all())
    assert bool((kv.k[0, table[0, 0]] != 0.5).any())  # the first sequence is fine
    kv.synchronize()  # cleared


@pytest.mark.parametrize("most", [2, 40], ids=["row by row", "by tiles"])
def test_append_of_a_first_sequence_that_does_not_start_at_zero(gpu, most):
    c = P.Cache(3, 1, 2, 64, PAGE, [most, 2], poison=0.5)
    kv = handle(c, 2)
    k = dev(draw(1, most + 2, 2, 64))
    kv.append(0, k, k, dev(c.table), dev(c.lens), dev(np.array([1, most, most + 2], np.int32)))
    with pytest.raises(U.UadError) as e:
        kv.synchronize()
    assert e.value.status == 9
    pages = c.table[0][c.table[0] >= 0].tolist()
    assert bool((kv.k[0, pages] == 0.5).all()) and bool((kv.v[0, pages] == 0.5).all())


@pytest.mark.parametrize("lens,wide", [([60, 65, 40], 4), ([60, -1, 40], 4), ([60, 1281, 40], 80), ([1281] + [20] * 70, 80)])
def test_attend_takes_a_length_that_it_cannot_use_for_none(gpu, lens, wide):
    """Narrow tables (a workgroup per unit) and wide ones, planned by a wave's lanes and by the whole workgroup."""
    fine = [n if 0 <= n <= 16 * wide else 0 for n in lens]
    c = P.Cache(6, 1, 1, 64, PAGE, fine, wide=wide)
    c.fill(2)
    kv = handle(c, 2)
    table = np.where(c.table < 0, 0, c.table).astype(np.int32)
    q = draw(1, len(lens), 2, 64)
    got = kv.attend(0, dev(q), dev(table), dev(np.array(lens, np.int32)))
    with pytest.raises(U.UadError) as e:
        kv.synchronize()
    assert e.value.status == 9
    check_attend(c, kv, 0, q, got, 0, False)  # the others' results, and zeros


@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf")])
def test_an_infinity_enters_its_own_outputs_only(gpu, where, bad):
    """Of a key: all of its sequence's head; of a value: that column.  They need not be finite, the others are as ever."""
    lens = [700, 50, 70]
    outs = []
    q = dev(draw(1, 3, 4, 64))
    for value in (0.25, bad):
        c = P.Cache(9, 1, 2, 64, PAGE, lens)
        c.fill(4)
        pg, off = c.slot(0, 57)
        (c.k[0, pg, 1, off] if where == "k" else c.v[0, pg, 1, :, off])[3] = value
        kv = handle(c, 4)
        outs.append(kv.attend(0, q, dev(c.table), dev(c.lens)).cpu())
        kv.synchronize()
    want, got = outs
    assert torch.equal(got[1:], want[1:]) and torch.equal(got[0, :2], want[0, :2])
    if where == "v":
        assert not bool(got[0, 2:, 3].isfinite().any())
        got[0, 2:, 3] = want[0, 2:, 3]
        assert torch.equal(got, want)
