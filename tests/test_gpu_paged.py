"""The paged K/V cache on the GPU against its definition in 64 bits: append with rotation, attention of one token, the
expert's prefix from pages, and a decoding run of them together.  Slots that no token holds are NaN throughout, and page
table entries behind a sequence's last page are no pages."""
import dataclasses
import math

import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
import uad_workloads as W
from tests import paged_oracle as P
from tests.harness import log

pytestmark = pytest.mark.gpu
BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)) if isinstance(a, np.ndarray) else a
    return t.to("cuda") if dtype is None else t.to("cuda", dtype)


def handle(c, heads, max_seqs=None, rope=0, pairs=False, theta=10000.0, stream=None):
    return U.PagedKV(c.layers, heads, c.hkv, c.hd, c.page, c.n_pages, max_seqs or max(1, len(c.lens)), dtype=c.dtype,
                     rope_dim=rope, rope_theta=theta, rope_pairs=pairs, k_scale=c.scales[0], v_scale=c.scales[1],
                     k=dev(c.k), v=dev(c.v), stream=stream)


def draw(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def offset_by_one(t):
    """The same values, one element past a 16-byte boundary."""
    buf = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    out = buf[1:].view(t.shape)
    out.copy_(t)
    return out


def bits(t):
    return t.view(torch.uint8 if t.element_size() == 1 else torch.int16).cpu().numpy()


# ------------------------------------------------------------------------------------------------------- append
def check_append(c, kv, layer, k, v, new, after, row_start, rope, pairs, positions=None, theta=10000.0):
    """The pools of `kv` after the append of rows k, v: every new slot near its exact value, every other bit as it was."""
    want_k, want_v = bits(c.k).copy(), bits(c.v).copy()
    got_k, got_v = kv.k.cpu(), kv.v.cpu()
    bk, bv = bits(got_k), bits(got_v)
    fk, fv = got_k.double().numpy(), got_v.double().numpy()
    worst = 0.0
    for b, n in enumerate(new):
        for j in range(n):
            r = row_start[b] + j
            pos = after[b] - n + j
            pg, off = c.slot(b, pos)
            turn = pos if positions is None else int(positions[r])
            ek, size = P.rotate(k[r:r + 1].double().numpy(), [turn], rope, pairs, theta)
            ev = v[r:r + 1].double().numpy()
            for e, s, got, scale in ((ek[0], size[0], fk[layer, pg, :, off], c.scales[0]),
                                     (ev[0], 0 * ev[0], fv[layer, pg, :, :, off], c.scales[1])):
                cut = np.clip(e, -448 * scale, 448 * scale) if c.dtype == F8 else e
                ratio = np.abs(got - cut / scale) / np.maximum(P.append_bound(cut, s, scale, c.dtype), 1e-300)
                assert np.all(ratio <= 1), (b, j, float(ratio.max()))
                worst = max(worst, float(ratio.max()))
            want_k[layer, pg, :, off] = bk[layer, pg, :, off]
            want_v[layer, pg, :, :, off] = bv[layer, pg, :, :, off]
    assert np.array_equal(want_k, bk) and np.array_equal(want_v, bv), "a slot that no row goes to changed"
    return worst


APPENDS = [
    # hkv, hd, page, new rows, lengths before, given, cache, rope, pairs
    (1, 64, 16, [1], [0], BF16, BF16, 64, False),
    (1, 256, 16, [1], [816], BF16, BF16, 256, False),
    (2, 128, 32, [1, 1, 1], [0, 31, 32], F32, F8, 64, True),
    (3, 64, 64, [1] * 70, list(range(70)), BF16, F8, 0, False),
    (1, 256, 16, [33, 0, 1, 16, 0], [0, 5, 15, 16, 7], BF16, BF16, 256, True),
    (2, 128, 256, [300, 2, 255], [250, 255, 1], F32, BF16, 128, False),
    (5, 64, 32, [0, 65, 0, 0, 31, 64], [3, 31, 0, 9, 33, 64], BF16, F8, 32, False),
    (4, 128, 128, [130, 127], [127, 1], F32, F8, 16, True),
    (1, 64, 64, [513], [1], BF16, BF16, 48, False),
    (8, 256, 64, [70, 3], [60, 64], BF16, F8, 256, False),
    (1, 64, 16, [2] * 130, [i % 37 for i in range(130)], F32, BF16, 64, False),
    (16, 64, 16, [40], [7], F32, BF16, 64, True),
    (2, 64, 16, [i % 11 for i in range(130)], [i * 13 % 37 for i in range(130)], BF16, F8, 64, False),
    (1, 128, 64, [i % 23 for i in range(65)], [i * 13 % 70 for i in range(65)], F32, BF16, 128, True),
    (1, 256, 128, [1, 200, 64, 65], [127, 128, 64, 63], BF16, F8, 0, False),
    (1, 64, 32, [8, 8], [30, 31], BF16, BF16, 64, False),
    (1, 64, 32, [7, 8], [30, 31], BF16, BF16, 64, False),
    (1, 64, 16, [9 if i % 3 else 0 for i in range(600)], [i % 40 for i in range(600)], BF16, BF16, 64, False),
    (1, 64, 16, [17] * 70 + [0] * 200 + [400], [i % 40 for i in range(271)], BF16, F8, 64, False),
    (1, 256, 64, [70, 9], [3, 60], BF16, BF16, 160, False),
    (1, 256, 64, [70, 9], [3, 60], F32, F8, 48, True),
    (2, 128, 32, [3, 1], [30, 31], BF16, F8, 48, False),
    (1, 64, 16, [2 if i % 7 == 0 else i % 2 for i in range(4200)], [0] * 4200, BF16, BF16, 64, False),
    (2, 64, 16, [5 + i % 17 for i in range(67)], [i * 13 % 37 for i in range(67)], BF16, F8, 64, False),
]


@pytest.mark.parametrize("i", range(len(APPENDS)))
def test_append(gpu, i):
    hkv, hd, page, new, before, given, cache, rope, pairs = APPENDS[i]
    after = [a + b for a, b in zip(new, before)]
    c = P.Cache(i, 2, hkv, hd, page, after, cache=cache)
    kv = handle(c, hkv, rope=rope, pairs=pairs)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    total = int(starts[-1])
    k, v = (draw(10 * i + j, total, hkv, hd).to(given) for j in range(2))
    single = all(n == 1 for n in new)
    kv.append(1, dev(k), dev(v), dev(c.table), dev(c.lens), None if single else dev(starts))
    kv.synchronize()
    worst = check_append(c, kv, 1, k, v, new, after, starts, rope, pairs)
    if single:  # the same with explicit starts
        first = bits(kv.k), bits(kv.v)
        kv.append(1, dev(k), dev(v), dev(c.table), dev(c.lens), dev(starts))
        kv.synchronize()
        assert np.array_equal(first[0], bits(kv.k)) and np.array_equal(first[1], bits(kv.v))
    log(f"[append {i}] worst error {worst:.2f} of its bound")


@pytest.mark.parametrize("given,cache,hd,page", [(BF16, BF16, 128, 16), (F32, F8, 64, 64), (F32, BF16, 256, 32), (BF16, F8, 256, 128)])
@pytest.mark.parametrize("form", ["slices", "offset", "odd rows"])
def test_append_strides_and_padding_rows(gpu, given, cache, hd, page, form):
    """Rows that are slices of wider ones, that start off a 16-byte boundary or lie an odd distance apart; rows of NaN
    behind the last sequence are ignored."""
    hkv, new, before = 2, [40, 1, 0, 23], [3, 0, 8, 41]
    after = [a + b for a, b in zip(new, before)]
    c = P.Cache(5, 1, hkv, hd, page, after, cache=cache)
    kv = handle(c, hkv, rope=hd)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = int(starts[-1]) + 9
    k, v = (draw(7 + j, rows, hkv, hd).to(given) for j in range(2))
    k[starts[-1]:] = v[starts[-1]:] = float("nan")
    extra = 1 if form == "odd rows" else 32
    wide = torch.full((2, rows, 2 * hkv * hd + extra), 9.0, dtype=given, device="cuda")
    kd, vd = (wide[j, :, hkv * hd:2 * hkv * hd].unflatten(1, (hkv, hd)) for j in range(2))
    kd.copy_(dev(k)), vd.copy_(dev(v))
    if form == "offset":
        kd, vd = offset_by_one(dev(k)), offset_by_one(dev(v))
    kv.append(0, kd, vd, dev(c.table), dev(c.lens), dev(starts))
    kv.synchronize()
    check_append(c, kv, 0, k, v, new, after, starts, hd, False)


@pytest.mark.parametrize("second", [40, 2])  # by tiles and row by row
def test_append_positions(gpu, second):
    """Rotation positions of the caller's, far ones and negative ones among them; base 500000."""
    hkv, hd, page, new = 1, 128, 32, [5, second]
    c = P.Cache(8, 1, hkv, hd, page, new)
    kv = handle(c, hkv, rope=128, theta=500000.0)
    starts = np.array([0, 5, 5 + second], np.int32)
    positions = np.concatenate([[0, 1, -3, 2 ** 31 - 1, -2 ** 31], 1000003 * np.arange(second) + 7]).astype(np.int32)
    k, v = draw(1, 5 + second, hkv, hd), draw(2, 5 + second, hkv, hd)
    kv.append(0, dev(k), dev(v), dev(c.table), dev(c.lens), dev(starts), dev(positions))
    kv.synchronize()
    check_append(c, kv, 0, k, v, new, new, starts, 128, False, positions, 500000.0)


@pytest.mark.parametrize("n", [1, 50])
def test_append_values_beyond_the_8_bit_range(gpu, n):
    """Cut to +-448 of a step; infinities too; a NaN stays one."""
    c = P.Cache(2, 1, 1, 64, 16, [n], cache=F8)
    kv = handle(c, 1)
    k = torch.zeros((n, 1, 64))
    vals = torch.tensor([1e30, -1e30, math.inf, -math.inf, 448 * 0.03, 460 * 0.03, 1e-9, -0.0])
    k[0, 0, :8] = vals
    k[0, 0, 8] = math.nan
    kv.append(0, dev(k), dev(k), dev(c.table), dev(c.lens), dev(np.array([0, n], np.int32)))
    kv.synchronize()
    pg = int(c.table[0, 0])
    got = kv.k[0, pg, 0, 0].float().cpu()
    assert got[:8].tolist() == [448, -448, 448, -448, 448, 448, 0, 0]
    assert math.isnan(float(got[8])) and math.isnan(float(kv.v[0, pg, 0, 8, 0].float()))


BAD_APPENDS = {  # lens, starts, a change of the page table (or none), of 3 sequences with rows 2, 1, 20
    "length below zero": ([-1, 1, 20], [0, 2, 3, 23], None),
    "length beyond the table": ([2, 1000, 20], [0, 2, 3, 23], None),
    "length below the new rows": ([2, 1, 19], [0, 2, 3, 23], None),
    "page below zero": ([2, 1, 20], [0, 2, 3, 23], (2, 1, -1)),
    "page beyond the pool": ([2, 1, 20], [0, 2, 3, 23], (0, 0, 1 << 30)),
    "starts fall": ([3, 2, 21], [0, 3, 2, 23], None),
    "starts beyond the rows": ([2, 1, 21], [0, 2, 3, 24], None),
    "starts below zero": ([2, 1, 20], [-2, 2, 3, 23], None),
    "no row belongs to the first": ([2, 1, 20], [1, 2, 3, 23], None),
}


@pytest.mark.parametrize("what", BAD_APPENDS)
@pytest.mark.parametrize("rows", [30, 2])  # by tiles and row by row
def test_append_reports_what_it_cannot_use(gpu, what, rows):
    lens, starts, page = BAD_APPENDS[what]
    less = 20 - rows
    lens, starts = lens[:2] + [lens[2] - less], starts[:3] + [starts[3] - less]
    if page and page[0] == 2:
        page = (2, 1 if rows > 16 else 0, page[2])
    c = P.Cache(3, 1, 2, 64, 16, [2, 1, rows], poison=0.5)
    kv = handle(c, 2)
    table = c.table.copy()
    if page:
        table[page[0], page[1]] = page[2]
    k = dev(draw(1, 3 + rows, 2, 64))
    kv.append(0, k, k, dev(table), dev(np.array(lens, np.int32)), dev(np.array(starts, np.int32)))
    with pytest.raises(U.UadError) as e:
        kv.synchronize()
    assert e.value.status == 9
    kv.synchronize()  # cleared
    # pages of no sequence are as they were
    spare = sorted(set(range(c.n_pages)) - set(c.table[c.table >= 0].tolist()))
    assert spare and bool((kv.k[0, spare] == 0.5).all()) and bool((kv.v[0, spare] == 0.5).all())
    kv.append(0, k, k, dev(c.table), dev(c.lens), dev(np.array([0, 2, 3, 3 + rows], np.int32)))
    kv.synchronize()


# ------------------------------------------------------------------------------------------------------- attend
def check_attend(c, kv, layer, q, got, rope, pairs, positions=None, scale=None, theta=10000.0):
    scale = 1 / math.sqrt(c.hd) if scale is None else scale
    positions = c.lens.astype(np.int64) - 1 if positions is None else positions
    o, b, a = P.attend(c, layer, q.double().numpy(), positions, rope, pairs, scale, theta)
    n = np.maximum(c.lens, 1)[:, None, None]
    f32 = q.dtype == F32
    bound = P.attend_bound(o, b, n, c.hd, a, 3 if f32 else 2, 3 if f32 else 2, q.dtype)
    err = np.abs(got.double().cpu().numpy() - o)
    empty = c.lens == 0
    assert np.all(err[empty] == 0)
    ratio = err[~empty] / np.maximum(bound[~empty], 1e-300)
    assert np.all(ratio <= 1), float(ratio.max())
    return float(ratio.max()) if ratio.size else 0.0


ATTENDS = [
    # hkv, group, hd, page, lengths, q, cache, rope, pairs
    (1, 1, 64, 16, [1], BF16, BF16, 0, False),
    (1, 8, 256, 16, [817], BF16, BF16, 256, False),
    (1, 8, 256, 16, [816, 0, 1, 15, 16, 17, 31, 32, 33], F32, BF16, 256, False),
    (2, 6, 128, 32, [64, 65, 63, 127, 128, 129, 0, 700], BF16, F8, 128, True),
    (4, 1, 64, 64, [5, 200, 1, 64], F32, F8, 32, False),
    (3, 16, 64, 128, [300, 1, 128, 129], BF16, BF16, 64, False),
    (1, 17, 128, 16, [100, 33], F32, BF16, 0, False),
    (2, 40, 64, 32, [90, 257], BF16, F8, 16, True),
    (8, 4, 128, 256, [1000, 3], BF16, BF16, 128, False),
    (1, 1, 256, 32, [5000], F32, F8, 256, False),
    (1, 4, 128, 64, [9000, 1, 0, 77], BF16, BF16, 128, False),
    (1, 2, 64, 16, [i * 7 % 90 for i in range(150)], BF16, BF16, 64, False),
    (5, 3, 64, 16, [0, 0, 0], BF16, F8, 64, False),
    (16, 1, 64, 16, [40] * 9, F32, BF16, 64, False),
    (1, 5, 256, 64, [20000], BF16, F8, 256, False),
    (1, 1, 64, 16, [(i * 37) % 120 for i in range(700)], F32, BF16, 64, False),
    (2, 6, 128, 32, [5000, 900, 64, 0, 1281], BF16, F8, 128, False),
    (2, 4, 64, 16, [3000, 1, 700, 640, 641], F32, BF16, 64, True),
    (1, 3, 256, 128, [256, 257, 2100, 0], F32, F8, 0, False),
    (3, 20, 128, 16, [1500, 384, 385], BF16, BF16, 64, True),
    (2, 1, 64, 16, [(i * 37) % 50 for i in range(1300)] + [3000], BF16, F8, 0, False),
    (1, 2, 128, 32, [30] * 80 + [4000] + [1] * 20 + [0] * 30, BF16, BF16, 128, False),
]


@pytest.mark.parametrize("i", range(len(ATTENDS)))
def test_attend(gpu, i):
    hkv, group, hd, page, lens, given, cache, rope, pairs = ATTENDS[i]
    c = P.Cache(i, 2, hkv, hd, page, lens, cache=cache)
    c.fill(i, 1)
    heads = hkv * group
    kv = handle(c, heads, rope=rope, pairs=pairs)
    q = (1.5 * draw(i, len(lens), heads, hd)).to(given)
    got = kv.attend(1, dev(q), dev(c.table), dev(c.lens))
    kv.synchronize()
    worst = check_attend(c, kv, 1, q, got, rope, pairs)
    again = kv.attend(1, dev(q), dev(c.table), dev(c.lens))
    assert torch.equal(got, again)
    log(f"[attend {i}] worst error {worst:.2f} of its bound")


def test_attend_peaked_scores(gpu):
    """Scores of hundreds: the running maximum rises at every step, falls never."""
    for spread, lens in ((60.0, [700, 33]), (8.0, [257, 64])):
        c = P.Cache(4, 1, 1, 64, 16, lens)
        c.fill(9, spread=spread)
        for b, n in enumerate(lens):  # later keys larger: the maximum moves all along
            for pos in range(n):
                pg, off = c.slot(b, pos)
                c.k[0, pg, :, off] = (c.k[0, pg, :, off].float() * (pos + 1) / n).to(BF16)
        kv = handle(c, 4)
        q = draw(3, 2, 4, 64)
        got = kv.attend(0, dev(q), dev(c.table), dev(c.lens))
        check_attend(c, kv, 0, q, got, 0, False)


def test_attend_positions_and_scale(gpu):
    c = P.Cache(4, 1, 2, 128, 32, [77, 140])
    c.fill(4)
    kv = handle(c, 4, rope=128, theta=1e6)
    q = draw(3, 2, 4, 128)
    positions = np.array([123456789, -5], np.int32)
    for scale in (0.5, 0.0, -0.1):
        got = kv.attend(0, dev(q), dev(c.table), dev(c.lens), positions=dev(positions), scale=scale)
        kv.synchronize()
        check_attend(c, kv, 0, q, got, 128, False, positions, scale, 1e6)


@pytest.mark.parametrize("given", [BF16, F32])
def test_attend_slices_and_offsets(gpu, given):
    """Queries that are a slice of a fused projection's output, results into a slice, both off 16-byte boundaries."""
    hkv, group, hd = 2, 4, 64
    c = P.Cache(6, 1, hkv, hd, 16, [50, 1, 33])
    c.fill(2)
    kv = handle(c, hkv * group, rope=64)
    q = draw(1, 3, 8, 64).to(given)
    ref = kv.attend(0, dev(q), dev(c.table), dev(c.lens))
    check_attend(c, kv, 0, q, ref, 64, False)
    for extra in (8, 7, 1):
        wide = torch.full((2, 3, 512 + 2 * extra), 7.0, dtype=given, device="cuda")
        qv, ov = (wide[j, :, extra:extra + 512].unflatten(1, (8, 64)) for j in range(2))
        qv.copy_(dev(q))
        kv.attend(0, qv, dev(c.table), dev(c.lens), out=ov)
        assert torch.equal(ov, ref)
        assert bool((wide[1, :, :extra] == 7).all()) and bool((wide[1, :, extra + 512:] == 7).all())


def test_attend_shared_pages_and_fewer_sequences(gpu):
    """Two sequences read the same pages; a call with fewer sequences than the handle was made for."""
    c = P.Cache(6, 1, 1, 64, 16, [60, 50, 40, 9], shared=(0, 1, 2))
    c.fill(2)
    kv = handle(c, 2, max_seqs=300)
    q = draw(1, 4, 2, 64)
    got = kv.attend(0, dev(q), dev(c.table), dev(c.lens))
    check_attend(c, kv, 0, q, got, 0, False)
    part = kv.attend(0, dev(q)[:2], dev(c.table)[:2].contiguous(), dev(c.lens)[:2].contiguous())
    c.lens = c.lens[:2]
    check_attend(c, kv, 0, q[:2], part, 0, False)


@pytest.mark.parametrize("what,lens,page", [("length below zero", [60, -1, 40], None), ("beyond the table", [60, 50, 10 ** 6], None),
                                            ("page below zero", [60, 50, 40], (1, 2, -1)), ("page beyond", [60, 50, 40], (0, 0, 1000))])
def test_attend_reports_what_it_cannot_use(gpu, what, lens, page):
    c = P.Cache(6, 1, 1, 64, 16, [60, 50, 40])
    c.fill(2)
    kv = handle(c, 2)
    q = draw(1, 3, 2, 64)
    table = c.table.copy()
    if what == "beyond the table":
        table[table < 0] = 0  # what is cut to the table is read
    if page:
        table[page[0], page[1]] = page[2]
    kv.attend(0, dev(q), dev(table), dev(np.array(lens, np.int32)))
    with pytest.raises(U.UadError) as e:
        kv.synchronize()
    assert e.value.status == 9
    got = kv.attend(0, dev(q), dev(c.table), dev(c.lens))
    kv.synchronize()
    check_attend(c, kv, 0, q, got, 0, False)


def test_offsets_beyond_32_bits(gpu):
    """Pools of over 2^32 bytes and 2^31 elements: the last pages."""
    hkv, hd, page = 8, 256, 64
    n_pages = 2 ** 31 // (hkv * hd * page) + 40
    kv = U.PagedKV(1, 8, hkv, hd, page, n_pages, 1, rope_dim=256)
    n = 150
    c = P.Cache(1, 1, hkv, hd, page, [n])
    far = np.array([[n_pages - 1, 3, n_pages - 2]], np.int32)
    k, v = (draw(j, n, hkv, hd).to(BF16) for j in range(2))
    kv.append(0, dev(k), dev(v), dev(far), dev(c.lens), dev(np.array([0, n], np.int32)))
    kv.synchronize()
    near = torch.from_numpy(c.table[0, :3].astype(np.int64))
    c.k[0, near], c.v[0, near] = kv.k[0, far[0].tolist()].cpu(), kv.v[0, far[0].tolist()].cpu()
    starts, got_k = [0], c.k.clone()
    ek, size = P.rotate(k.double().numpy(), range(n), 256, False)
    tok = c.tokens(0, 0)
    assert np.all(np.abs(tok[0] - ek) <= P.append_bound(ek, size, 1.0, BF16)) and np.array_equal(tok[1], v.double().numpy())
    q = draw(5, 1, 8, hd).to(BF16)
    got = kv.attend(0, dev(q), dev(far), dev(c.lens))
    kv.synchronize()
    check_attend(c, kv, 0, q, got, 256, False)


# ------------------------------------------------------------------------------------------------------- together
def decode_inputs(seqs, heads, hkv, hd, layers, steps):
    return [[tuple(draw(100 * t + 10 * l + j, seqs, h, hd).to(BF16) for j, h in enumerate((heads, hkv, hkv))) for l in range(layers)]
            for t in range(steps)]


def run_decode(kv, table, lens, steps):
    outs = []
    for step in steps:
        lens += 1
        for l, (q, k, v) in enumerate(step):
            kv.append(l, k, v, table, lens)
            outs.append(kv.attend(l, q, table, lens))
    return outs


def test_decoding_run_and_the_experts_prefix(gpu):
    """A prompt into the cache, four tokens decoded behind it, then the expert's prefix from the pages: the step is the
    one that uad_set_prefix_kv gives for the same values, bit for bit."""
    wl = dataclasses.replace(W.get_workload("tiny"), batch=3, chunk=5, prefix=40)
    s = wl.shape
    seqs, heads, hkv, hd, L = 3, 8, s.n_kv_heads, s.head_dim, s.n_layers
    prompt = [37, 50, 41]
    after = [n + 4 for n in prompt]
    c = P.Cache(1, L, hkv, hd, 16, after)
    kv = handle(c, heads, rope=hd)
    starts = np.concatenate([[0], np.cumsum(prompt)]).astype(np.int32)
    table, lens = dev(c.table), dev(np.array(prompt, np.int32))
    for l in range(L):
        k, v = (dev(draw(l * 2 + j, int(starts[-1]), hkv, hd).to(BF16)) for j in range(2))
        kv.append(l, k, v, table, lens, dev(starts))
    steps = [[tuple(dev(x) for x in layer) for layer in step] for step in decode_inputs(seqs, heads, hkv, hd, L, 4)]
    outs = run_decode(kv, table, lens, steps)
    kv.synchronize()
    assert lens.tolist() == after
    c.k, c.v = kv.k.cpu(), kv.v.cpu()
    for l in range(L):  # the last step's outputs of each layer against what the pages hold
        check_attend(c, kv, l, steps[-1][l][0].cpu(), outs[-L + l], hd, False)
    weights = W.make_weights(wl)
    x0 = np.stack([W.make_noise(wl, b) for b in range(3)])
    t, dt = (np.full((3, 5), f, np.float32) for f in (0.5, -0.1))
    dense = [np.stack([np.stack([c.tokens(l, b, 40)[j] for b in range(3)]) for l in range(L)]).astype(np.float32) for j in range(2)]
    got = []
    ex = U.ActionExpert(s, 4, 5, 70)
    try:
        ex.load_weights(weights)
        for source in ("dense", "paged"):
            ones = torch.ones((L, 4, 70, hkv, hd), device="cuda")
            ex.set_prefix_kv(ones, ones, 4, 70)
            if source == "dense":
                ex.set_prefix_kv(dense[0], dense[1], 3, 40)
            else:
                ex.set_prefix_paged(kv, table, lens, 40)
            x, vel = dev(x0), torch.empty((3, 5, 7), device="cuda")
            ex.step(x, dev(t), dev(dt), torch.zeros((3, 5), dtype=torch.uint8, device="cuda"), vel)
            ex.synchronize()
            got.append((x.cpu().numpy().tobytes(), vel.cpu().numpy().tobytes()))
        assert got[0] == got[1]
    finally:
        ex.close()


@pytest.mark.parametrize("hd,hkv,page,prefix,cache", [(64, 4, 16, 33, BF16), (128, 2, 64, 64, F8), (256, 1, 32, 1, BF16), (64, 2, 256, 0, F8),
                                                      (256, 1, 128, 130, F8), (128, 1, 16, 95, BF16)])
def test_prefix_from_pages_on_two_streams(gpu, hd, hkv, page, prefix, cache):
    """The cache on its own stream: the prefix waits for its appends, and later appends for the prefix."""
    shape = W.ModelShape(2, 128, max(4, hkv), hkv, hd, 256, 7)
    wl = dataclasses.replace(W.get_workload("tiny"), shape=shape, batch=2, chunk=3, prefix=prefix)
    c = P.Cache(2, 2, hkv, hd, page, [prefix + 5, max(prefix, 1)], cache=cache)
    c.fill(3)
    tok = [[c.tokens(l, b, prefix) for b in range(2)] for l in range(2)]
    dense = [np.array([[tok[l][b][j] for b in range(2)] for l in range(2)], np.float32).reshape(2, 2, prefix, hkv, hd) for j in range(2)]
    ex = U.ActionExpert(shape, 3, 3, prefix + 40)
    side = torch.cuda.Stream()
    got = []
    try:
        ex.load_weights(W.make_weights(wl))
        x0 = np.stack([W.make_noise(wl, b) for b in range(2)])
        t, dt, mask = (dev(np.full((2, 3), f, d)) for f, d in ((0.5, np.float32), (-0.1, np.float32), (0, np.uint8)))
        for source in ("dense", "paged"):
            if source == "dense":
                ex.set_prefix_kv(dense[0], dense[1], 2, prefix)
            else:
                torch.cuda.synchronize()
                with torch.cuda.stream(side):
                    kv = handle(c, hkv, stream=side)
                    table, lens = dev(c.table), dev(c.lens)
                    rows = dev(draw(4, prefix + 5, hkv, hd))
                    side.synchronize()
                    ex.set_prefix_paged(kv, table, lens, prefix)
                    # overwrites what the prefix was read from
                    starts = dev(np.array([0, prefix + 5, prefix + 5], np.int32))
                    for l in range(2):
                        kv.append(l, rows, rows, table, lens, starts)
            x, vel = dev(x0), torch.empty((2, 3, 7), device="cuda")
            ex.step(x, t, dt, mask, vel)
            ex.synchronize()
            got.append((x.cpu().numpy().tobytes(), vel.cpu().numpy().tobytes()))
        kv.synchronize()
        assert got[0] == got[1]
    finally:
        ex.close()


def test_prefix_from_pages_reports_short_sequences_and_bad_pages(gpu):
    shape = W.ModelShape(2, 128, 4, 2, 64, 256, 7)
    c = P.Cache(2, 2, 2, 64, 16, [40, 40], poison=0.0)
    c.fill(3)
    kv = handle(c, 2)
    ex = U.ActionExpert(shape, 2, 3, 64)
    try:
        bad = c.table.copy()
        bad[1, 1] = c.n_pages
        for table, lens in ((c.table, [40, 39]), (bad, [40, 40]), (c.table, [40, -1])):
            ex.set_prefix_paged(kv, dev(table), dev(np.array(lens, np.int32)), 40)
            for h in (ex, kv):
                with pytest.raises(U.UadError) as e:
                    h.synchronize()
                assert e.value.status == 9
                h.synchronize()
        ex.set_prefix_paged(kv, dev(c.table), dev(c.lens), 40)
        ex.synchronize(), kv.synchronize()
    finally:
        ex.close()


def test_decoding_step_in_a_graph(gpu):
    """Captured once, replayed with other lengths, tokens and tables; eager work between the replays."""
    seqs, heads, hkv, hd, L = 3, 8, 2, 128, 2
    start = [30, 400, 0]
    c = P.Cache(1, L, hkv, hd, 16, [n + 6 for n in start])
    c.lens = np.array(start, np.int32)
    c.fill(3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        kv, ref = (handle(c, heads, rope=hd, stream=side) for _ in range(2))
        table, lens, lens_ref = dev(c.table), dev(c.lens), dev(c.lens)
        steps = [[tuple(dev(x) for x in layer) for layer in step] for step in decode_inputs(seqs, heads, hkv, hd, L, 4)]
        ins = [tuple(torch.zeros_like(x) for x in layer) for layer in steps[0]]
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs = run_decode(kv, table, lens, [ins])
        for step in steps:
            for dst, src in zip(ins, step):
                for d_, s_ in zip(dst, src):
                    d_.copy_(s_)
            graph.replay()
            want = run_decode(ref, table, lens_ref, [step])
            side.synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b)
            assert torch.equal(lens, lens_ref)
        assert np.array_equal(bits(kv.k), bits(ref.k)) and np.array_equal(bits(kv.v), bits(ref.v))
        kv.synchronize(), ref.synchronize()


def test_two_handles_at_once(gpu):
    """Handles of their own on two streams share pools and run at the same time; every result is the one of a lone call."""
    hkv, group, hd = 2, 4, 128
    c = P.Cache(9, 2, hkv, hd, 16, [700, 90, 0, 1500], cache=BF16)
    c.fill(4)
    pools = dev(c.k), dev(c.v)
    streams = [torch.cuda.Stream() for _ in range(2)]
    table, lens = dev(c.table), dev(c.lens)
    kvs = [U.PagedKV(2, hkv * group, hkv, hd, 16, c.n_pages, 4, rope_dim=hd, k=pools[0], v=pools[1], stream=s) for s in streams]
    qs = [dev(draw(i, 4, hkv * group, hd)) for i in range(2)]
    alone = [[kvs[i].attend(l, qs[i], table, lens) for l in range(2)] for i in range(2)]
    for kv in kvs:
        kv.synchronize()
    for i in range(2):
        check_attend(c, kvs[i], 1, qs[i].cpu(), alone[i][1], hd, False)
    outs = [[torch.empty_like(qs[i]) for _ in range(40)] for i in range(2)]
    torch.cuda.synchronize()
    for n in range(40):
        for i in range(2):
            kvs[i].attend(n % 2, qs[i], table, lens, out=outs[i][n])
    torch.cuda.synchronize()
    for i in range(2):
        for n in range(40):
            assert torch.equal(outs[i][n], alone[i][n % 2])


def test_what_a_call_allocates_is_its_streams(gpu):
    """Freed memory that another stream's queued work may still use is not taken for pools and outputs."""
    c = P.Cache(9, 1, 1, 64, 16, [300])
    c.fill(4)
    side = torch.cuda.Stream()
    q, table, lens, k, v = dev(draw(1, 1, 4, 64)), dev(c.table), dev(c.lens), dev(c.k), dev(c.v)
    want = handle(c, 4).attend(0, q, table, lens)
    torch.cuda.synchronize()
    olds = [torch.empty_like(x) for x in (q, k, v)]
    used = {x.data_ptr() for x in olds}
    del olds
    kv = U.PagedKV(1, 4, 1, 64, 16, c.n_pages, 1, dtype=c.dtype, k_scale=c.scales[0], v_scale=c.scales[1], stream=side)
    with torch.cuda.stream(side):
        kv.k.copy_(k), kv.v.copy_(v)
    out = kv.attend(0, q, table, lens)
    assert not used & {out.data_ptr(), kv.k.data_ptr(), kv.v.data_ptr()}
    kv.synchronize()
    assert torch.equal(out, want)


def test_status_is_reported_once_each_time(gpu):
    """Clearing the status does not clear what work queued right after it raises."""
    c = P.Cache(9, 1, 1, 64, 16, [40])
    c.fill(4)
    side = torch.cuda.Stream()
    kv = handle(c, 4, stream=side)
    q, bad, lens = dev(draw(1, 1, 4, 64)), dev(np.full_like(c.table, -1)), dev(c.lens)
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    for _ in range(50):
        kv.attend(0, q, bad, lens, out=out)
        with pytest.raises(U.UadError) as e:
            kv.synchronize()
        assert e.value.status == 9
    kv.synchronize()


def test_another_stream_and_a_closed_handle(gpu):
    c = P.Cache(9, 1, 1, 64, 16, [300])
    c.fill(4)
    kv = handle(c, 4)
    q, table, lens = dev(draw(1, 1, 4, 64)), dev(c.table), dev(c.lens)
    want = kv.attend(0, q, table, lens)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    kv.set_stream(side)
    with torch.cuda.stream(side):
        out = torch.zeros_like(q)
        kv.attend(0, q, table, lens, out=out)
        got = out + 0  # ordered behind it on that stream
    kv.synchronize()
    assert torch.equal(got, want)
    for _ in range(5):  # destroyed with work queued: waits for it
        kv.attend(0, q, table, lens, out=out)
    kv.close()
    assert torch.equal(out, want)
    with pytest.raises(U.UadError):
        kv.attend(0, q, table, lens)
    with pytest.raises(U.UadError):
        kv.synchronize()


def test_values_of_the_cache_that_are_not_finite(gpu):
    """A NaN among a sequence's own keys and values makes its outputs NaN (an infinity may), and nobody else's."""
    c = P.Cache(9, 1, 1, 64, 16, [100, 50, 70])
    c.fill(4)
    want = handle(c, 2).attend(0, dev(draw(1, 3, 2, 64)), dev(c.table), dev(c.lens))
    for where, bad in (("k", math.nan), ("k", math.inf), ("v", math.nan)):
        d = P.Cache(9, 1, 1, 64, 16, [100, 50, 70])
        d.fill(4)
        pg, off = d.slot(0, 57)
        if where == "k":
            d.k[0, pg, 0, off, 3] = bad
        else:
            d.v[0, pg, 0, :, off] = bad
        kv = handle(d, 2)
        got = kv.attend(0, dev(draw(1, 3, 2, 64)), dev(d.table), dev(d.lens))
        kv.synchronize()
        assert torch.equal(got[1:], want[1:])
        assert bad == math.inf or bool(got[0].isnan().all())


def test_prompt_and_prefix_in_a_graph(gpu):
    """A new prompt into the pages and the expert's prefix from them, captured once and replayed with other rows, lengths
    and tables; the steps between the replays are those of the same values handed over densely."""
    shape = W.ModelShape(2, 128, 4, 2, 64, 256, 7)
    wl = dataclasses.replace(W.get_workload("tiny"), shape=shape, batch=2, chunk=3, prefix=40)
    side = torch.cuda.Stream()
    ex = U.ActionExpert(shape, 2, 3, 40, stream=side)
    ref = U.ActionExpert(shape, 2, 3, 40)
    try:
        ex.load_weights(W.make_weights(wl)), ref.load_weights(W.make_weights(wl))
        c = P.Cache(3, 2, 2, 64, 16, [50, 41])
        x0 = np.stack([W.make_noise(wl, b) for b in range(2)])
        t, dt, mask = (dev(np.full((2, 3), f, d)) for f, d in ((0.5, np.float32), (-0.1, np.float32), (0, np.uint8)))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            kv = handle(c, 2, rope=64, stream=side)
            table, lens, starts = dev(c.table), dev(c.lens), dev(np.array([0, 50, 91], np.int32))
            rows = torch.zeros((2, 2, 91, 2, 64), dtype=BF16, device="cuda")
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                for l in range(2):
                    kv.append(l, rows[0, l], rows[1, l], table, lens, starts)
                ex.set_prefix_paged(kv, table, lens, 40)
            for n in range(3):
                rows.copy_(dev(draw(n, 2, 2, 91, 2, 64).to(BF16)))
                table.copy_(dev(np.where(c.table >= 0, np.roll(np.arange(c.n_pages), n)[np.maximum(c.table, 0)], -1).astype(np.int32)))
                graph.replay()
                x, vel = dev(x0), torch.empty((2, 3, 7), device="cuda")
                ex.step(x, t, dt, mask, vel)
                ex.synchronize(), kv.synchronize()
                d = P.Cache(3, 2, 2, 64, 16, [50, 41])
                d.k, d.v, d.table = kv.k.cpu(), kv.v.cpu(), table.cpu().numpy()
                dense = [np.stack([np.stack([d.tokens(l, b, 40)[j] for b in range(2)]) for l in range(2)]).astype(np.float32) for j in range(2)]
                # what the pages hold is what was appended
                ek, size = P.rotate(rows[0, 1, 50:90].double().cpu().numpy(), range(40), 64, False)
                assert np.all(np.abs(dense[0][1, 1] - ek) <= P.append_bound(ek, size, 1.0, BF16))
                ref.set_prefix_kv(dense[0], dense[1], 2, 40)
                y, want = dev(x0), torch.empty((2, 3, 7), device="cuda")
                torch.cuda.synchronize()
                ref.step(y, t, dt, mask, want)
                ref.synchronize()
                assert torch.equal(vel, want) and torch.equal(x, y)
    finally:
        ex.close(), ref.close()


def test_empty_calls(gpu):
    c = P.Cache(1, 1, 1, 64, 16, [4, 5], poison=0.25)
    kv = handle(c, 2)
    none = torch.empty((0, 1, 64), device="cuda")
    kv.append(0, none, none, dev(c.table), dev(c.lens), dev(np.zeros(3, np.int32)))
    empty = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    no_lens = torch.empty((0,), dtype=torch.int32, device="cuda")
    kv.append(0, none, none, empty, no_lens)
    assert kv.attend(0, torch.empty((0, 2, 64), device="cuda"), empty, no_lens).shape == (0, 2, 64)
    # every row is behind the last sequence
    rows = torch.full((7, 1, 64), float("nan"), device="cuda")
    kv.append(0, rows, rows, dev(c.table), dev(c.lens), dev(np.zeros(3, np.int32)))
    kv.synchronize()
    assert bool((kv.k == 0.25).all()) and bool((kv.v == 0.25).all())


def test_binding_refuses(gpu):
    c = P.Cache(1, 1, 2, 64, 16, [4, 5])
    kv = handle(c, 4)
    rows, q = torch.zeros((2, 2, 64), device="cuda"), torch.zeros((2, 4, 64), device="cuda")
    table, lens = dev(c.table), dev(c.lens)
    ok = dict(layer=0, k=rows, v=rows, page_table=table, lens=lens)
    for change in (dict(k=rows.cpu()), dict(k=rows.half()), dict(k=rows.bfloat16()), dict(k=rows[:, :1]), dict(v=rows[:1]),
                   dict(k=rows.transpose(1, 2)), dict(k=rows[:1].expand(2, 2, 64)), dict(page_table=table.long()),
                   dict(page_table=table[0]), dict(lens=lens[:1]), dict(lens=lens.cpu()), dict(row_start=lens),
                   dict(positions=lens[:1]), dict(page_table=table.t().contiguous().t())):
        with pytest.raises(ValueError):
            kv.append(**{**ok, **change})
    for change in (dict(layer=1), dict(layer=-1)):
        with pytest.raises(U.UadError):
            kv.append(**{**ok, **change})
    for change in (dict(out=q[:1]), dict(out=q.bfloat16()), dict(q=q[:1]), dict(positions=lens[:1])):
        with pytest.raises(ValueError):
            kv.attend(**{**dict(layer=0, q=q, page_table=table, lens=lens), **change})
    with pytest.raises(U.UadError):
        kv.attend(0, q, table, lens, scale=float("nan"))
    with pytest.raises(U.UadError) as e:  # a pool that ends early is refused by the library as well
        U.uad_kv_create(1, 4, 2, 64, 16, 10 ** 6, 2, U.UAD_DTYPE_BF16, 0, 0, 1.0, 1.0, 1.0, kv.k, kv.v)
    assert e.value.status == 2
    kv.synchronize()
