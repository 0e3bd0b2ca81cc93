"""Attention of new rows over the paged cache with queries large enough for the kernel of many rows: units cut into splits
of their tiles, units whole, columns shared by two waves and not; against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
from tests import rows_oracle as R
from tests.harness import log
from tests.test_gpu_paged import BF16, F32, F8, dev, draw, offset_by_one
from tests.test_gpu_paged_rows import ODD, check, handle, made, starts_of

pytestmark = pytest.mark.gpu

MANY = [
    # hkv, group, hd, page, new rows, lengths, given, cache, rope, pairs, window, sinks, causal
    (8, 4, 128, 64, [64], [2000], BF16, BF16, 128, False, 0, 0, True),
    (8, 4, 128, 16, [64, 3], [1500, 700], BF16, "blocks", 128, False, 0, 0, True),
    (2, 4, 256, 32, [130], [900], F32, BF16, 256, False, 0, 0, True),
    (1, 8, 256, 64, [150], [700], BF16, F8, 128, True, 300, 5, False),
    (8, 4, 64, 64, [130], [3000], F32, "blocks", 64, False, 0, 0, True),
    (8, 4, 64, 128, [100, 0, 33], [1100, 50, 33], BF16, BF16, 64, False, 500, 70, True),
    (6, 3, 64, 16, [250], [260], BF16, F8, 32, True, 0, 0, True),
    (1, 5, 128, 32, [450], [460], BF16, BF16, 128, False, 0, 0, False),
    (1, 5, 128, 32, [450], [460], F32, F8, 128, False, 1, 0, True),
    (1, 8, 256, 16, [1, 160], [5000, 160], BF16, BF16, 256, False, 0, 0, True),
    (1, 8, 256, 16, [140], [1500], F32, "blocks", 0, False, 40, 3, False),
    (8, 4, 64, 16, [i % 13 for i in range(130)], [i % 13 + 37 * i % 400 for i in range(130)], BF16, BF16, 64, False, 33, 2, True),
    (8, 4, 64, 16, [i % 13 for i in range(130)], [i % 13 + (3000 if i == 77 else 5) for i in range(130)], F32, "blocks", 64, False, 0, 0, True),
    (16, 16, 64, 16, [130], [150], BF16, BF16, 64, False, 9, 2, True),
    (16, 16, 64, 64, [131], [400], BF16, "blocks", 64, False, 0, 0, True),
    (16, 16, 64, 32, [130], [190], F32, F8, 64, True, 0, 0, False),
    (16, 16, 128, 32, [140], [200], F32, "blocks", 128, False, 0, 0, True),
    (16, 16, 128, 16, [150], [170], BF16, BF16, 128, True, 70, 9, False),
    (16, 16, 128, 64, [100, 41], [164, 41], BF16, F8, 128, False, 0, 0, True),
    (16, 16, 256, 64, [129, 1], [129, 300], BF16, F8, 256, False, 0, 0, False),
    (16, 16, 256, 16, [130], [131], F32, F8, 256, False, 20, 3, True),
    (16, 16, 256, 32, [130], [140], F32, BF16, 256, False, 0, 0, True),
    # sequences beyond a thread each, heads beyond a unit's columns
    (2, 16, 64, 16, [1 + i % 2 for i in range(1100)], [1 + i % 2 + i * 7 % 50 for i in range(1100)], BF16, BF16, 64, False, 0, 0, True),
    (2, 16, 128, 16, [i % 4 for i in range(700)], [i % 4 + (900 if i == 650 else i % 9) for i in range(700)], BF16, "blocks", 128, False, 20, 3, True),
    (1, 16, 256, 16, [2 + i % 2 for i in range(600)], [3 + i % 30 for i in range(600)], F32, BF16, 64, True, 0, 0, False),
    (4, 16, 64, 16, [8 + i % 3 for i in range(70)], [10 + i * 11 % 130 for i in range(70)], BF16, "blocks", 64, False, 0, 0, True),
    (1, 200, 128, 16, [31], [500], BF16, BF16, 128, False, 0, 0, True),
    (2, 150, 64, 32, [17, 2], [300, 1000], F32, F8, 64, False, 100, 7, True),
]


@pytest.mark.parametrize("i", range(len(MANY)))
def test_attend_many_rows(gpu, i):
    hkv, group, hd, page, new, lens, given, cache, rope, pairs, window, sinks, causal = MANY[i]
    c = made(300 + i, hkv, hd, page, lens, cache)
    c.hide(new, window, sinks)
    kv = handle(c, hkv * group, rope=rope, pairs=pairs)
    q = (1.5 * draw(11 * i, sum(new), hkv * group, hd)).to(given)
    call = lambda: kv.attend_rows(0, dev(q), dev(c.table), dev(c.lens), dev(starts_of(new)), window=window, sinks=sinks, causal=causal)  # noqa: E731
    got = call()
    kv.synchronize()
    want = R.attend_rows(c, 0, q.double().numpy(), new, rope, pairs, 1 / math.sqrt(hd), window, sinks, causal)
    worst = check(got.double().cpu().numpy(), want, hd, given, i)
    again = call()
    kv.synchronize()
    assert torch.equal(got, again)  # the order of the sums does not depend on who comes first
    log(f"[attend_many_rows {i}] worst error {worst:.2f} of its bound")


# hkv, group, hd, rows, tokens before: two waves a column, whole and split; one wave
SIZES = [(8, 4, 64, 150, 40), (8, 4, 128, 64, 1100), (1, 8, 256, 140, 900), (16, 16, 64, 140, 40)]


@pytest.mark.parametrize("size", range(len(SIZES)))
@pytest.mark.parametrize("cache", [BF16, F8, "blocks"])
@pytest.mark.parametrize("window,sinks,causal", [(0, 0, True), (9, 2, True), (9, 20, False)])
def test_what_a_row_does_not_see_does_not_reach_it(gpu, size, cache, window, sinks, causal):
    """Keys and values that are not finite, here and there among the tokens, in one column of the head each: outputs are
    exact wherever no such token is seen, and NaN where a NaN among the values is."""
    hkv, group, hd, rows, before = SIZES[size]
    m = rows + before
    c = made(3, hkv, hd, 16, [m], cache)
    at = {m - 1: 3, m - 2: 5, m - rows // 2: 17, before - 5: 40, before + 3: 60, 1: 8}  # token: column
    for i, (x, col) in enumerate(at.items()):
        page, off = c.slot(0, x)
        c.v[0, page, 0, col, off] = ODD[i % 3 if cache == BF16 else 0]
    bad_key = m - 5
    page, off = c.slot(0, bad_key)
    c.k[0, page, 0, off, 11] = float("nan")
    kv = handle(c, hkv * group, rope=0)
    q = draw(2, rows, hkv * group, hd).to(BF16)
    got = kv.attend_rows(0, dev(q), dev(c.table), dev(c.lens), dev(starts_of([rows])), window=window, sinks=sinks, causal=causal)
    kv.synchronize()
    got = got.double().cpu().numpy()
    mask = R.sees(rows, m, window, sinks, causal)
    for x, col in at.items():  # the definition without them
        page, off = c.slot(0, x)
        c.v[0, page, 0, col, off] = 0.0
    page, off = c.slot(0, bad_key)
    c.k[0, page, 0, off, 11] = 0.0
    o, b, a, n = R.attend_rows(c, 0, q.double().numpy(), [rows], 0, False, 1 / math.sqrt(hd), window, sinks, causal)
    bound = R.rows_bound(o, b, n, hd, a, 2, BF16)
    free = np.ones((rows, hd), bool)  # outputs of the first KV head's that no odd value reaches
    for x, col in at.items():
        free[mask[:, x], col] = False
    free[mask[:, bad_key]] = False
    assert free.any() and not free.all()
    ok = np.abs(got - o) <= bound
    assert np.all(ok[:, group:])  # the other KV heads'
    own = got[:, :group]
    assert np.all(ok[:, :group] | ~free[:, None, :]), np.argwhere(~(ok[:, :group] | ~free[:, None, :]))[:5].tolist()
    for i, (x, col) in enumerate(at.items()):
        if cache != BF16 or i % 3 == 0:
            assert np.isnan(own[mask[:, x], :, col]).all()
        else:
            assert not np.isfinite(own[mask[:, x], :, col]).any()
    assert np.isnan(own[mask[:, bad_key]]).all()


@pytest.mark.parametrize("size", range(len(SIZES)))
def test_a_row_of_nan_is_the_only_one(gpu, size):
    hkv, group, hd, rows, before = SIZES[size]
    heads = hkv * group
    c = made(4, hkv, hd, 32, [rows + before, 6], BF16)
    kv = handle(c, heads, rope=hd)
    q = draw(8, rows + 6, heads, hd)
    q[rows // 2, 1, 30] = float("nan")
    got = kv.attend_rows(0, dev(q), dev(c.table), dev(c.lens), dev(starts_of([rows, 6])))
    kv.synchronize()
    got = got.double().cpu().numpy()
    assert np.isnan(got[rows // 2, 1]).all()
    q[rows // 2, 1, 30] = 0
    want = R.attend_rows(c, 0, q.double().numpy(), [rows, 6], hd, False, 1 / math.sqrt(hd))
    got[rows // 2, 1] = want[0][rows // 2, 1]
    check(got, want, hd, F32, "others")


@pytest.mark.parametrize("size", range(len(SIZES)))
def test_scores_far_apart(gpu, size):
    """Keys 60 times as large: softmax weights that vanish, maxima that rise from tile to tile and split to split."""
    hkv, group, hd, rows, before = SIZES[size]
    c = made(6, hkv, hd, 16, [rows + before], BF16, spread=60.0)
    c.k[0] *= torch.linspace(0.01, 1, c.n_pages)[torch.randperm(c.n_pages, generator=torch.Generator().manual_seed(1))].to(BF16)[:, None, None, None]
    kv = handle(c, hkv * group)
    q = draw(5, rows, hkv * group, hd)
    got = kv.attend_rows(0, dev(q), dev(c.table), dev(c.lens), dev(starts_of([rows])))
    kv.synchronize()
    want = R.attend_rows(c, 0, q.double().numpy(), [rows], 0, False, 1 / math.sqrt(hd))
    check(got.double().cpu().numpy(), want, hd, F32, "far")


@pytest.mark.parametrize("form", ["slices", "offset", "odd rows"])
@pytest.mark.parametrize("given,before", [(BF16, 30), (F32, 900)])
def test_strides_positions_and_padding_rows(gpu, form, given, before):
    hkv, group, hd, new = 8, 4, 64, [130, 0, 7]
    lens = [130 + before, 4, 7]
    c = made(9, hkv, hd, 16, lens, BF16)
    kv = handle(c, hkv * group, rope=hd, theta=500000.0)
    total, heads = sum(new) + 9, hkv * group
    q = draw(1, total, heads, hd).to(given)
    q[sum(new):] = float("nan")
    positions = np.concatenate([[0, 1, -3, 2 ** 31 - 1, -2 ** 31], 1000003 * np.arange(total - 5) + 7]).astype(np.int32)
    extra = 1 if form == "odd rows" else 32
    wide = torch.full((2, total, 3 * heads * hd + extra), 9.0, dtype=given, device="cuda")
    qd, out = (wide[j, :, heads * hd:2 * heads * hd].unflatten(1, (heads, hd)) for j in range(2))
    qd.copy_(dev(q))
    if form == "offset":
        qd, out = offset_by_one(dev(q)), offset_by_one(torch.full((total, heads, hd), 9.0, dtype=given, device="cuda"))
    kv.attend_rows(0, qd, dev(c.table), dev(c.lens), dev(starts_of(new)), out=out, positions=dev(positions), scale=0.3, window=800, sinks=3)
    kv.synchronize()
    want = R.attend_rows(c, 0, q[:sum(new)].double().numpy(), new, hd, False, 0.3, 800, 3, True, positions, 500000.0)
    check(out[:sum(new)].double().cpu().numpy(), want, hd, given, form)
    assert bool((out[sum(new):] == 9).all())
    if form != "offset":
        wide[1, :, heads * hd:2 * heads * hd] = 9
        assert bool((wide[1] == 9).all())


@pytest.mark.parametrize("what", ["page below zero", "page beyond the pool", "length beyond the table", "starts fall"])
def test_what_cannot_be_used_is_reported(gpu, what):
    """A bad page among a split unit's, a sequence that cannot be used between two that can."""
    new, lens = [70, 1, 70], [1000, 9, 1200]
    c = made(7, 8, 64, 16, lens, BF16)
    kv = handle(c, 32)
    table, starts = c.table.copy(), starts_of(new)
    lens = list(lens)
    if what.startswith("page"):
        table[0, 20] = -1 if "zero" in what else 1 << 30
    elif what.startswith("length"):
        lens[1] = 10 ** 6
    else:
        starts[2] = 60
    q = dev(draw(3, sum(new), 32, 64))
    out = torch.full_like(q, 7.0)
    kv.attend_rows(0, q, dev(table), dev(np.array(lens, np.int32)), dev(starts), out=out)
    with pytest.raises(U.UadError) as e:
        kv.synchronize()
    assert e.value.status == 9
    want = R.attend_rows(c, 0, q.double().cpu().numpy(), new, 0, False, 0.125)
    got = out.double().cpu().numpy()
    # starts of 0, 70, 60, 141 give rows 60 to 69 to two sequences
    fine = {"page": (71, 141), "length": (0, 70), "starts": (0, 60)}[what.split()[0]]
    check(got[slice(*fine)], tuple(x[slice(*fine)] for x in want), 64, F32, what)
    kv.attend_rows(0, q, dev(c.table), dev(c.lens), dev(starts_of(new)), out=out)  # the handle is as ever
    kv.synchronize()
    check(out.double().cpu().numpy(), want, 64, F32, "afterwards")


@pytest.mark.parametrize("cache", [BF16, "blocks"])
def test_a_captured_call_serves_any_lengths(gpu, cache):
    """One graph, replayed with other lengths and starts in the same arrays: other numbers of splits, units and sequences
    of a row, the program's own work between the replays."""
    rows = 160
    c = made(11, 8, 128, 32, [2000, 900], cache)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        kv = handle(c, 32, rope=128, stream=st)
        q, table, lens, starts = dev(draw(1, rows, 32, 128)), dev(c.table), dev(c.lens), dev(starts_of([rows - 1, 1]))
        out = torch.zeros_like(q)
        call = lambda o: kv.attend_rows(0, q, table, lens, starts, out=o)  # noqa: E731
        call(out)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            call(out)
        for new, after in (([rows - 1, 1], [2000, 900]), ([1, rows - 1], [5, 800]), ([0, 2], [0, 2]), ([rows, 0], [rows, 77]),
                           ([3, 1], [2000, 900]), ([80, 80], [1999, 81])):
            lens.copy_(dev(np.array(after, np.int32)))
            starts.copy_(dev(starts_of(new)))
            out.fill_(3)
            graph.replay()
            want = torch.full_like(q, 3)
            call(want)
            kv.synchronize()
            assert torch.equal(out, want) and bool((out[sum(new):] == 3).all()) and bool((out[:sum(new)] != 3).any())
            c.lens = np.array(after, np.int32)
            exact = R.attend_rows(c, 0, q[:sum(new)].double().cpu().numpy(), new, 128, False, 1 / math.sqrt(128))
            check(out[:sum(new)].double().cpu().numpy(), exact, 128, F32, (new, after))


def test_few_and_many_rows_in_turn(gpu):
    """The kernels share a handle's workspace and its counters: split calls of all of them, one after the other."""
    c = made(12, 8, 128, 64, [3000, 2500], BF16)
    kv = handle(c, 32, rope=128)
    q, table, lens = dev(draw(1, 140, 32, 128).to(BF16)), dev(c.table), dev(c.lens)
    calls = [lambda: kv.attend_rows(0, q, table, lens, dev(starts_of([70, 70]))), lambda: kv.attend_rows(0, q[:10], table, lens, dev(starts_of([9, 1]))),
             lambda: kv.attend(0, q[:2], table, lens), lambda: kv.attend_rows(0, q[:2], table, lens, window=2000)]
    first = [f() for f in calls]
    kv.synchronize()
    for _ in range(4):
        assert all(torch.equal(f(), x) for f, x in zip(calls, first))
    kv.synchronize()
    for f, new in ((first[0], [70, 70]), (first[1], [9, 1])):
        want = R.attend_rows(c, 0, q[:sum(new)].double().cpu().numpy(), new, 128, False, 1 / math.sqrt(128))
        check(f.double().cpu().numpy(), want, 128, BF16, new)
