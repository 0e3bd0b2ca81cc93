"""Wide heads with many query heads to a KV head: splits whose rows the join takes in more than one round, in one level
and in two, with a last run of heads that is shorter than the others."""
import pytest

from tests import paged_oracle as P
from tests.test_gpu_paged import BF16, F8, F32, check_attend, dev, draw, handle

pytestmark = pytest.mark.gpu

CASES = [
    # hkv, group, hd, page, lengths, q, cache, rope, pairs
    (1, 16, 256, 32, [2000, 300], F32, BF16, 256, False),
    (1, 9, 256, 16, [1, 255, 256, 257, 288, 0, 1100], BF16, BF16, 256, True),
    (1, 20, 256, 16, [20000], BF16, F8, 256, False),
    (2, 12, 256, 64, [9000, 3, 700], F32, F8, 64, True),
    (1, 27, 256, 128, [6000, 2500], BF16, BF16, 0, False),
    (1, 16, 256, 256, [40000], BF16, BF16, 256, False),
    (3, 16, 128, 16, [12000, 1, 2000], F32, F8, 128, False),
    (1, 13, 256, 64, [(i * 97) % 500 for i in range(70)] + [5000], BF16, F8, 256, False),
    (1, 33, 64, 16, [(i * 97) % 900 for i in range(66)] + [7000], F32, BF16, 64, False),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_attend_many_heads(gpu, i):
    hkv, group, hd, page, lens, given, cache, rope, pairs = CASES[i]
    c = P.Cache(40 + i, 1, hkv, hd, page, lens, cache=cache)
    c.fill(i)
    kv = handle(c, hkv * group, rope=rope, pairs=pairs)
    q = (1.5 * draw(i, len(lens), hkv * group, hd)).to(given)
    got = kv.attend(0, dev(q), dev(c.table), dev(c.lens))
    kv.synchronize()
    check_attend(c, kv, 0, q, got, rope, pairs)
