"""Attention of many new rows with as many units as workgroups run at once, some sequences long and others short: every row
is written, and the handle's later split calls are right too; against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
from tests import rows_oracle as R
from tests.test_gpu_paged import BF16, F32, dev, draw
from tests.test_gpu_paged_rows import check, handle, made, starts_of

pytestmark = pytest.mark.gpu

MIXES = [
    # hkv, group, hd, new rows, lengths, given
    (8, 4, 128, [10, 483], [3000, 483], BF16),
    (8, 4, 128, [10, 481], [3000, 481], F32),
    (8, 4, 128, [241, 241], [10000, 241], BF16),
    (1, 8, 256, [1, 2033], [4000, 2033], BF16),
    (8, 4, 64, [10, 995], [3000, 995], BF16),
    (4, 4, 128, [385, 609], [19200, 609], BF16),
    (8, 4, 128, [65, 65, 65, 257], [6000, 65, 65, 257], F32),
]


def call(kv, c, q, new):
    out = torch.full_like(q, float("nan"))
    kv.attend_rows(0, q, dev(c.table), dev(c.lens), dev(starts_of(new)), out=out)
    return out


@pytest.mark.parametrize("i", range(len(MIXES)))
def test_as_many_units_as_run_at_once(gpu, i):
    hkv, group, hd, new, lens, given = MIXES[i]
    c = made(40 + i, hkv, hd, 64, lens, BF16)
    kv = handle(c, hkv * group, rope=hd)
    q = (1.5 * draw(i, sum(new), hkv * group, hd)).to(given)
    got = call(kv, c, dev(q), new)
    # split calls of other numbers of rows afterwards, on the same handle
    others = [[64] + [0] * (len(new) - 1), [min(n, 20) for n in new], [1] * len(new)]
    later = [call(kv, c, dev(q[:sum(n)]), n) for n in others]
    kv.synchronize()
    for out, n in zip([got, *later], [new, *others]):
        want = R.attend_rows(c, 0, q[:sum(n)].double().numpy(), n, hd, False, 1 / math.sqrt(hd))
        check(out.double().cpu().numpy(), want, hd, given, n)


@pytest.mark.parametrize("hkv,group,hd,seqs,rows", [(8, 4, 128, 5, 200), (8, 4, 128, 5, 3), (1, 8, 256, 90, 100), (8, 4, 64, 90, 250), (2, 4, 64, 130, 2)])
def test_starts_that_fall_leave_the_handle_as_it_was(gpu, hkv, group, hd, seqs, rows):
    """Starts 0, n, 0, n, ..: every other sequence takes all of the call's rows, far more than it is launched for.  That is
    reported, and the handle's later split calls are right."""
    lens = [9000] + [rows] * (seqs - 1)
    c = made(60, hkv, hd, 64, lens, BF16)
    kv = handle(c, hkv * group, rope=hd)
    q = draw(3, rows + seqs + 8, hkv * group, hd).to(BF16)
    news = [[1 + 8 * (b == 0) for b in range(seqs)], [rows] + [0] * (seqs - 1)]
    before = [call(kv, c, dev(q[:sum(new)]), new) for new in news]
    kv.synchronize()
    starts = np.array([rows * (b % 2) for b in range(seqs + 1)], np.int32)
    guard = torch.full((rows + 2, hkv * group, hd), 7.0, dtype=BF16, device="cuda")
    kv.attend_rows(0, dev(q[:rows]), dev(c.table), dev(c.lens), dev(starts), out=guard[1:-1])
    with pytest.raises(U.UadError) as e:
        kv.synchronize()
    assert e.value.status == 9 and bool((guard[0] == 7).all()) and bool((guard[-1] == 7).all())
    for new, was in zip(news, before):
        out = call(kv, c, dev(q[:sum(new)]), new)
        kv.synchronize()
        assert torch.equal(out, was)
        want = R.attend_rows(c, 0, q[:sum(new)].double().numpy(), new, hd, False, 1 / math.sqrt(hd))
        check(out.double().cpu().numpy(), want, hd, BF16, new[:3])
