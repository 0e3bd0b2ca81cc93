"""Attention of new rows over the paged cache on the GPU against its definition in 64 bits: prompts, a few rows, single
tokens; windows, sinks, both directions; bf16 pools, 8-bit ones with one scale and with scales for blocks.  Slots that no
token holds and pages that no row sees are NaN throughout, and their page table entries are no pages."""
import math

import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
from tests import rows_oracle as R
from tests.harness import log
from tests.test_gpu_paged import BF16, F32, F8, dev, draw, offset_by_one

pytestmark = pytest.mark.gpu


def handle(c, heads, max_seqs=None, rope=0, pairs=False, theta=10000.0, stream=None):
    more = dict(block_scales=True, k_scales=dev(c.block[0]), v_scales=dev(c.block[1])) if c.blocks else dict(k_scale=c.scales[0], v_scale=c.scales[1])
    return U.PagedKV(c.layers, heads, c.hkv, c.hd, c.page, c.n_pages, max_seqs or max(1, len(c.lens)), dtype=c.dtype, rope_dim=rope,
                     rope_theta=theta, rope_pairs=pairs, k=dev(c.k), v=dev(c.v), stream=stream, **more)


def made(seed, hkv, hd, page, lens, cache, spread=1.0, **kw):
    c = R.Cache(seed, 1, hkv, hd, page, lens, blocks=cache == "blocks", cache=BF16 if cache == "blocks" else cache, **kw)
    c.fill(seed + 1, spread=spread)
    return c


def starts_of(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def check(out, want, hd, given, what):
    o, b, a, n = want
    ratio = np.abs(out - o) / np.maximum(R.rows_bound(o, b, n, hd, a, 3 if given == F32 else 2, given), 1e-300)
    worst = float(ratio.max()) if ratio.size else 0.0
    assert worst <= 1, (what, worst, np.argwhere(~(ratio <= 1))[:4].tolist())
    return worst


ROWS = [
    # hkv, group, hd, page, new rows (0: the form for single tokens), lengths, given, cache, rope, pairs, window, sinks, causal
    (1, 1, 64, 16, 0, [1], BF16, BF16, 64, False, 0, 0, True),
    (1, 8, 256, 16, 0, [0, 1, 17, 300], BF16, BF16, 256, False, 5, 2, True),
    (2, 4, 128, 32, 0, [1000, 3, 64, 65], F32, "blocks", 128, False, 33, 1, True),
    (1, 16, 64, 64, 0, [700, 0, 1], BF16, F8, 64, True, 64, 64, True),
    (2, 20, 64, 16, 0, [130, 50], F32, BF16, 32, False, 1, 0, True),
    (3, 5, 64, 16, 0, [i * 7 % 150 for i in range(130)], BF16, "blocks", 64, False, 17, 16, True),
    (1, 2, 64, 32, 0, [40000], F32, BF16, 64, False, 0, 0, True),          # joined in two levels
    (1, 2, 64, 32, 0, [30001, 9], BF16, "blocks", 64, False, 20000, 100, False),
    (1, 1, 64, 16, [1], [1], F32, BF16, 64, False, 0, 0, False),
    (1, 1, 64, 16, [16, 0, 17], [16, 9, 40], F32, BF16, 64, False, 0, 0, True),
    (2, 1, 128, 32, [33, 1], [33, 1], BF16, "blocks", 128, False, 0, 0, True),
    (1, 8, 256, 16, [50], [50], BF16, BF16, 256, False, 0, 0, False),
    (1, 8, 256, 64, [70, 3, 0, 0, 128], [70, 90, 0, 5, 300], F32, F8, 256, True, 0, 0, True),
    (2, 6, 128, 128, [100, 7], [260, 8], BF16, BF16, 64, False, 31, 3, True),
    (2, 3, 64, 256, [90, 31, 64], [400, 31, 65], F32, "blocks", 64, True, 16, 17, True),
    (1, 5, 64, 16, [129], [300], BF16, BF16, 64, False, 1, 0, True),
    (1, 5, 64, 16, [40], [300], BF16, "blocks", 0, False, 7, 200, False),
    (4, 1, 64, 32, [61, 2], [1061, 500], F32, BF16, 64, True, 100, 40, False),
    (1, 17, 64, 16, [3, 1, 2], [50, 1, 2], BF16, F8, 64, False, 0, 0, True),
    (1, 2, 64, 16, [i % 5 for i in range(200)], [i % 5 + i % 37 for i in range(200)], BF16, BF16, 64, False, 9, 2, True),
    (1, 4, 128, 64, [300], [2000], BF16, BF16, 128, False, 0, 0, True),
    (1, 4, 128, 64, [257], [257], F32, BF16, 128, False, 0, 0, True),
    (2, 2, 64, 64, [400, 131], [400, 700], BF16, "blocks", 64, False, 0, 0, True),
    (1, 8, 256, 32, [200], [333], BF16, "blocks", 256, False, 150, 10, True),
    (1, 3, 128, 16, [333, 5], [333, 1000], BF16, BF16, 128, True, 40, 5, False),
    (1, 1, 256, 128, [513], [700], F32, F8, 128, False, 0, 0, False),
    (2, 16, 64, 32, [65, 64, 63], [65, 64, 263], BF16, F8, 64, False, 0, 0, True),
    (1, 2, 128, 16, [2, 300, 1], [9000, 300, 1], BF16, BF16, 128, False, 0, 0, True),
]


@pytest.mark.parametrize("i", range(len(ROWS)))
def test_attend_rows(gpu, i):
    hkv, group, hd, page, new, lens, given, cache, rope, pairs, window, sinks, causal = ROWS[i]
    single = new == 0
    new = [1] * len(lens) if single else new
    c = made(100 + i, hkv, hd, page, lens, cache)
    c.hide(new, window, sinks)
    kv = handle(c, hkv * group, rope=rope, pairs=pairs)
    q = (1.5 * draw(7 * i, sum(new), hkv * group, hd)).to(given)
    starts = None if single else dev(starts_of(new))
    got = kv.attend_rows(0, dev(q), dev(c.table), dev(c.lens), starts, window=window, sinks=sinks, causal=causal)
    kv.synchronize()
    want = R.attend_rows(c, 0, q.double().numpy(), new, rope, pairs, 1 / math.sqrt(hd), window, sinks, causal)
    worst = check(got.double().cpu().numpy(), want, hd, given, i)
    if single and all(n > 0 for n in lens):  # the same with explicit starts
        again = kv.attend_rows(0, dev(q), dev(c.table), dev(c.lens), dev(starts_of(new)), window=window, sinks=sinks, causal=causal)
        assert torch.equal(got, again)
    again = kv.attend_rows(0, dev(q), dev(c.table), dev(c.lens), starts, window=window, sinks=sinks, causal=causal)
    kv.synchronize()
    assert torch.equal(got, again)  # the order of the sums does not depend on who comes first
    log(f"[attend_rows {i}] worst error {worst:.2f} of its bound")


@pytest.mark.parametrize("given,cache,hd", [(BF16, BF16, 256), (F32, "blocks", 128), (BF16, F8, 64)])
def test_a_single_token_is_what_attend_gives(gpu, given, cache, hd):
    lens = [300, 1, 64, 0, 4097]
    c = made(5, 2, hd, 32, lens, cache)
    kv = handle(c, 8, rope=hd)
    q = dev((1.5 * draw(3, 5, 8, hd)).to(given))
    a, b = kv.attend(0, q, dev(c.table), dev(c.lens)), kv.attend_rows(0, q, dev(c.table), dev(c.lens))
    kv.synchronize()
    assert torch.equal(a, b) and not bool(b[3].any())
    want = R.attend_rows(c, 0, q.double().cpu().numpy(), [1] * 5, hd, False, 1 / math.sqrt(hd))
    check(a.double().cpu().numpy(), want, hd, given, "attend")


@pytest.mark.parametrize("rows", [20, 200])
@pytest.mark.parametrize("form", ["slices", "offset", "odd rows"])
@pytest.mark.parametrize("given", [BF16, F32])
def test_strides_positions_and_padding_rows(gpu, rows, form, given):
    """Rows that are slices of wider ones, off a 16-byte boundary or an odd distance apart; far positions of the caller's;
    rows behind the last sequence are not looked at and their outputs stay."""
    hkv, group, hd, new, lens = 2, 3, 64, [rows, 0, 7], [rows + 30, 4, 7]
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
    kv.attend_rows(0, qd, dev(c.table), dev(c.lens), dev(starts_of(new)), out=out, positions=dev(positions), scale=0.3, window=50, sinks=3)
    kv.synchronize()
    want = R.attend_rows(c, 0, q[:sum(new)].double().numpy(), new, hd, False, 0.3, 50, 3, True, positions, 500000.0)
    check(out[:sum(new)].double().cpu().numpy(), want, hd, given, form)
    assert bool((out[sum(new):] == 9).all())
    if form != "offset":
        wide[1, :, heads * hd:2 * heads * hd] = 9
        assert bool((wide[1] == 9).all())


ODD = [float("nan"), float("inf"), -float("inf")]


@pytest.mark.parametrize("rows", [24, 150])
@pytest.mark.parametrize("cache", [BF16, F8, "blocks"])
@pytest.mark.parametrize("window,sinks,causal", [(0, 0, True), (9, 2, True), (9, 20, False)])
def test_what_a_row_does_not_see_does_not_reach_it(gpu, rows, cache, window, sinks, causal):
    """Keys and values that are not finite, here and there among the tokens, in one column of the head each: outputs are
    exact wherever no such token is seen, and NaN where a NaN among the values is."""
    hkv, group, hd, m = 1, 4, 64, rows + 40
    c = made(3, hkv, hd, 16, [m], cache)
    at = {m - 1: 3, m - 2: 5, m - rows // 2: 17, 25: 40, 33: 60, 1: 8}  # token: column
    for i, (x, col) in enumerate(at.items()):
        page, off = c.slot(0, x)
        c.v[0, page, 0, col, off] = ODD[i % 3 if cache == BF16 else 0]
    bad_key = m - 5
    page, off = c.slot(0, bad_key)
    c.k[0, page, 0, off, 11] = float("nan")
    kv = handle(c, hkv * group, rope=0)
    q = draw(2, rows, group, hd).to(BF16)
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
    free = np.ones((rows, hd), bool)  # outputs that no odd value reaches
    for x, col in at.items():
        free[mask[:, x], col] = False
    free[mask[:, bad_key]] = False
    assert free.any() and not free.all()
    ok = np.abs(got - o) <= bound
    assert np.all(ok | ~free[:, None, :]), np.argwhere(~(ok | ~free[:, None, :]))[:5].tolist()
    for i, (x, col) in enumerate(at.items()):
        if cache != BF16 or i % 3 == 0:
            assert np.isnan(got[mask[:, x], :, col]).all()
        else:
            assert not np.isfinite(got[mask[:, x], :, col]).any()
    assert np.isnan(got[mask[:, bad_key]]).all()


@pytest.mark.parametrize("rows", [5, 300])
def test_a_row_of_nan_is_the_only_one(gpu, rows):
    c = made(4, 1, 128, 32, [rows + 20, 6], BF16)
    kv = handle(c, 4, rope=128)
    q = draw(8, rows + 6, 4, 128)
    q[rows // 2, 1, 30] = float("nan")
    got = kv.attend_rows(0, dev(q), dev(c.table), dev(c.lens), dev(starts_of([rows, 6])))
    kv.synchronize()
    got = got.double().cpu().numpy()
    assert np.isnan(got[rows // 2, 1]).all()
    q[rows // 2, 1, 30] = 0
    want = R.attend_rows(c, 0, q.double().numpy(), [rows, 6], 128, False, 1 / math.sqrt(128))
    got[rows // 2, 1] = want[0][rows // 2, 1]
    check(got, want, 128, F32, "others")


@pytest.mark.parametrize("rows", [9, 280])
def test_scores_far_apart(gpu, rows):
    """Keys 60 times as large: softmax weights that vanish, maxima that rise from tile to tile."""
    c = made(6, 1, 64, 16, [rows + 200], BF16, spread=60.0)
    c.k[0] *= torch.linspace(0.01, 1, c.n_pages)[torch.randperm(c.n_pages, generator=torch.Generator().manual_seed(1))].to(BF16)[:, None, None, None]
    kv = handle(c, 2)
    q = draw(5, rows, 2, 64)
    got = kv.attend_rows(0, dev(q), dev(c.table), dev(c.lens), dev(starts_of([rows])))
    kv.synchronize()
    check(got.double().cpu().numpy(), R.attend_rows(c, 0, q.double().numpy(), [rows], 0, False, 0.125), 64, F32, "far")


BAD = {  # of 3 sequences with 2, 1, rows rows: a length of another, starts, a change of the page table; who is wrong
    "length below zero": ((0, -1), None, None, [0]),
    "length beyond the table": ((1, 100000), None, None, [1]),
    "length below the rows": ((1, 0), None, None, [1]),
    "page below zero": (None, None, (2, 1, -1), [2]),
    "page beyond the pool": (None, None, (0, 0, 1 << 30), [0]),
    "starts fall": (None, [0, 3, 2, None], None, [1]),
    "starts beyond the rows": (None, [0, 2, 3, 9999], None, [2]),
    "no row belongs to the first": (None, [1, 2, 3, None], None, [0]),
}


@pytest.mark.parametrize("what", BAD)
@pytest.mark.parametrize("rows", [30, 300])
def test_what_cannot_be_used_is_reported(gpu, what, rows):
    length, starts, page, wrong = BAD[what]
    base = [40, 9, rows + 20]
    lens = list(base)
    if length:
        lens[length[0]] = length[1]
    starts = [s if s is not None else 3 + rows for s in starts or [0, 2, 3, None]]
    c = made(7, 1, 64, 16, base, BF16)
    kv = handle(c, 2)
    table = c.table.copy()
    if page:
        table[page[0], page[1]] = page[2]
    q = dev(draw(3, 3 + rows, 2, 64))
    out = torch.full_like(q, 7.0)
    kv.attend_rows(0, q, dev(table), dev(np.array(lens, np.int32)), dev(np.array(starts, np.int32)), out=out)
    with pytest.raises(U.UadError) as e:
        kv.synchronize()
    assert e.value.status == 9
    kv.synchronize()  # once
    if page is None:  # the others are as ever
        fine = [b for b in range(3) if b not in wrong]
        want = R.attend_rows(c, 0, q.double().cpu().numpy(), [2, 1, rows], 0, False, 0.125)
        for b in fine:
            if starts[b + 1] - starts[b] == [2, 1, rows][b] and starts[b] == [0, 2, 3][b]:
                s = slice(starts[b], starts[b + 1])
                check(out[s].double().cpu().numpy(), tuple(x[s] for x in want), 64, F32, what)
        for b in wrong:
            lo, hi = [0, 2, 3][b], [2, 3, 3 + rows][b]
            own = [r for r in range(lo, hi) if not any(starts[f] <= r < starts[f + 1] for f in fine)]
            assert bool((out[own] == 7).all())


def test_bad_lengths_of_single_tokens_give_zeros(gpu):
    c = made(7, 1, 64, 16, [40, 9, 20], BF16)
    kv = handle(c, 2)
    q = dev(draw(3, 3, 2, 64))
    got = kv.attend_rows(0, q, dev(c.table), dev(np.array([-3, 9, 10 ** 6], np.int32)), window=4)
    with pytest.raises(U.UadError):
        kv.synchronize()
    assert not bool(got[0].any()) and not bool(got[2].any())
    want = R.attend_rows(c, 0, q.double().cpu().numpy(), [1, 1, 1], 0, False, 0.125, 4)
    check(got[1:2].double().cpu().numpy(), tuple(x[1:2] for x in want), 64, F32, "the fine one")


def test_two_handles_on_two_streams(gpu):
    """Handles that share pools, each on its own stream, at once; and a call that comes from another stream."""
    c = made(8, 1, 128, 32, [3000, 500], BF16)
    s = [torch.cuda.Stream() for _ in range(2)]
    a = handle(c, 4, rope=128, stream=s[0])
    b = U.PagedKV(1, 4, 1, 128, 32, c.n_pages, 2, rope_dim=128, k=a.k, v=a.v, stream=s[1])
    q, table, lens = dev(draw(1, 200, 4, 128)), dev(c.table), dev(c.lens)
    starts = dev(starts_of([190, 10]))
    torch.cuda.synchronize()
    outs = []
    for _ in range(8):
        outs.append(a.attend_rows(0, q, table, lens, starts))
        outs.append(b.attend_rows(0, q, table, lens, starts))
        outs.append(a.attend_rows(0, q[:2], table, lens, window=40))
    a.synchronize(), b.synchronize()
    want = R.attend_rows(c, 0, q.double().cpu().numpy(), [190, 10], 128, False, 1 / math.sqrt(128))
    check(outs[0].double().cpu().numpy(), want, 128, F32, "streams")
    assert all(torch.equal(x, outs[i % 3 if i % 3 == 2 else 0]) for i, x in enumerate(outs))


@pytest.mark.parametrize("rows,cache", [(3, BF16), (200, BF16), (200, "blocks")])
def test_a_captured_call_serves_any_lengths(gpu, rows, cache):
    """One graph, replayed with other lengths and starts in the same arrays, the program's own work between the replays."""
    c = made(11, 1, 128, 32, [2000, 900], cache)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        kv = handle(c, 4, rope=128, stream=st)
        q, table, lens, starts = dev(draw(1, rows, 4, 128)), dev(c.table), dev(c.lens), dev(starts_of([rows - 1, 1]))
        out = torch.zeros_like(q)
        call = lambda o: kv.attend_rows(0, q, table, lens, starts, out=o, window=700, sinks=5)  # noqa: E731
        call(out)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            call(out)
        for new, after in (([rows - 1, 1], [2000, 900]), ([1, rows - 1], [5, 800]), ([0, 2], [0, 2]), ([rows, 0], [rows, 77])):
            lens.copy_(dev(np.array(after, np.int32)))
            starts.copy_(dev(starts_of(new)))
            out.fill_(3)
            graph.replay()
            want = torch.full_like(q, 3)
            call(want)
            kv.synchronize()
            assert torch.equal(out, want) and bool((out[sum(new):] == 3).all()) and bool((out[:sum(new)] != 3).any())
