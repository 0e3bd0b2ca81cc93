"""Attention of many new rows over 8-bit pools, whose calls reach the kernel of many rows from larger queries on than those
over bf16 pools: the tests of test_gpu_paged_many_rows with such."""
import math

import pytest
import torch

from tests import rows_oracle as R
from tests import test_gpu_paged_many_rows as M
from tests.test_gpu_paged import BF16, F32, F8, dev, draw
from tests.test_gpu_paged_rows import check, handle, made, starts_of

pytestmark = pytest.mark.gpu

MANY = [
    # hkv, group, hd, page, new rows, lengths, given, cache, rope, pairs, window, sinks, causal
    (8, 4, 128, 64, [200], [2000], BF16, "blocks", 128, False, 0, 0, True),
    (8, 4, 128, 16, [170, 3], [1500, 700], F32, F8, 128, False, 0, 0, True),
    (2, 4, 128, 32, [700, 60], [900, 1000], BF16, "blocks", 64, True, 300, 5, False),
    (1, 5, 128, 32, [1100], [1110], F32, "blocks", 128, False, 0, 0, False),
    (1, 5, 128, 16, [1100], [1300], BF16, F8, 128, False, 1, 0, True),
    (8, 4, 64, 64, [260], [3000], F32, "blocks", 64, False, 0, 0, True),
    (8, 4, 64, 128, [250, 0, 33], [1100, 50, 33], BF16, F8, 64, False, 500, 70, True),
    (6, 3, 64, 16, [450], [460], BF16, "blocks", 32, True, 0, 0, True),
    (2, 150, 64, 32, [25, 2], [300, 1000], F32, F8, 64, False, 100, 7, True),
    (1, 200, 128, 16, [31], [500], BF16, "blocks", 128, False, 0, 0, True),
    # sequences beyond a thread each
    (8, 4, 128, 64, [5 + i % 17 for i in range(130)], [5 + i % 17 + (3000 if i == 77 else 5) for i in range(130)], BF16, "blocks", 128, False, 33, 2, True),
    (2, 16, 128, 16, [3 + i % 4 for i in range(700)], [3 + i % 4 + (900 if i == 650 else i % 9) for i in range(700)], BF16, "blocks", 128, False, 20, 3, True),
    (8, 4, 64, 16, [9 + i % 13 for i in range(130)], [9 + i % 13 + (3000 if i == 77 else 5) for i in range(130)], F32, "blocks", 64, False, 0, 0, True),
]


@pytest.mark.parametrize("i", range(len(MANY)))
def test_attend_many_rows(gpu, i):
    hkv, group, hd, page, new, lens, given, cache, rope, pairs, window, sinks, causal = MANY[i]
    c = made(500 + i, hkv, hd, page, lens, cache)
    c.hide(new, window, sinks)
    kv = handle(c, hkv * group, rope=rope, pairs=pairs)
    q = (1.5 * draw(13 * i, sum(new), hkv * group, hd)).to(given)
    call = lambda: kv.attend_rows(0, dev(q), dev(c.table), dev(c.lens), dev(starts_of(new)), window=window, sinks=sinks, causal=causal)  # noqa: E731
    got, again = call(), call()
    kv.synchronize()
    want = R.attend_rows(c, 0, q.double().numpy(), new, rope, pairs, 1 / math.sqrt(hd), window, sinks, causal)
    check(got.double().cpu().numpy(), want, hd, given, i)
    assert torch.equal(got, again)


# as there, of queries large enough for 8-bit pools
SIZES = [(8, 4, 64, 260, 40), (8, 4, 128, 170, 1100)]


@pytest.mark.parametrize("size", range(len(SIZES)))
@pytest.mark.parametrize("cache", [F8, "blocks"])
@pytest.mark.parametrize("window,sinks,causal", [(0, 0, True), (9, 2, True), (9, 20, False)])
def test_what_a_row_does_not_see_does_not_reach_it(gpu, monkeypatch, size, cache, window, sinks, causal):
    monkeypatch.setattr(M, "SIZES", SIZES)
    M.test_what_a_row_does_not_see_does_not_reach_it(gpu, size, cache, window, sinks, causal)
