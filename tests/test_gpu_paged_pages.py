"""Page tables on the GPU against the same in plain Python, and a run of the paged cache's calls together: pages taken, a
prompt and its attention, decoding with a window in a captured step that takes and gives back pages, the expert's prefix."""
import math

import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
from tests import rows_oracle as R
from tests.test_gpu_paged import BF16, F8, dev, draw
from tests.test_gpu_paged_rows import starts_of

pytestmark = pytest.mark.gpu
I32 = torch.int32


class Tables:
    """The calls' arrays on the GPU beside the model of them in plain Python."""

    def __init__(self, seed, page, n_pages, seqs, wide, max_seqs=None):
        self.kv = U.PagedKV(1, 1, 1, 64, page, n_pages, max_seqs or seqs, dtype=F8)
        ids = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
        table = np.full((seqs, wide), -1, np.int32)
        self.m = R.Pages(page, n_pages, table, [0] * seqs, ids)
        self.table, self.lens, self.free = dev(table), dev(np.zeros(seqs, np.int32)), dev(ids)
        self.n_free = dev(np.array([n_pages], np.int32))
        self.starts = torch.full((seqs + 1,), -5, dtype=I32, device="cuda")

    def same(self):
        n = len(self.m.free)
        return (self.table.tolist() == self.m.table and self.lens.tolist() == self.m.lens and self.n_free.tolist() == [n]
                and self.free[:n].tolist() == self.m.free)

    def reserve(self, new, n_rows=None, **kw):
        slots = torch.full((sum(new) if n_rows is None else n_rows,), -5, dtype=torch.int64, device="cuda")
        self.kv.reserve(self.lens, self.table, self.free, self.n_free, dev(np.array(new, np.int32)), self.starts, slots, **kw)
        return slots


SIZES = [  # page, seqs, most new tokens, rounds
    (16, 1, 1, 40), (16, 3, 50, 6), (64, 64, 300, 4), (32, 65, 40, 4), (16, 300, 9, 5), (128, 1000, 3, 3), (16, 2, 9000, 2), (256, 5, 1, 4)]


@pytest.mark.parametrize("i", range(len(SIZES)))
def test_reserve_and_release(gpu, i):
    page, seqs, most, rounds = SIZES[i]
    r = np.random.default_rng(i)
    wide = -(-most * rounds // page) + 2
    t = Tables(i, page, seqs * wide, seqs, wide)
    for k in range(rounds):
        new = [int(x) for x in r.integers(0, most + 1, seqs)]
        padding = int(r.integers(0, 4))
        slots = t.reserve(new, sum(new) + padding)
        starts, want = t.m.reserve(new)
        assert t.starts.tolist() == starts and slots.tolist() == want + [-1] * padding and t.same()
        if k == rounds // 2:  # some have gone
            gone = [b for b in range(seqs) if b % 3 == 0]
            t.lens[dev(np.array(gone))] = 0
            for b in gone:
                t.m.lens[b] = 0
            window, sinks = 0, 0
        else:
            window, sinks = int(r.integers(1, 2 * page)), int(r.integers(0, 2 * page))
        t.kv.release(t.lens, t.table, t.free, t.n_free, window, sinks)
        t.m.release(window, sinks)
        assert t.same()
        if k < rounds // 2:  # shorter again: the pages behind go back
            cut = [int(x) for x in r.integers(0, 4, seqs)]
            t.m.lens = [max(0, m - c) for m, c in zip(t.m.lens, cut)]
            t.lens.copy_(dev(np.array(t.m.lens, np.int32)))
            t.kv.release(t.lens, t.table, t.free, t.n_free)
            t.m.release(0, 0)
            assert t.same()
    t.kv.synchronize()


def test_one_token_each_without_counts_starts_and_slots(gpu):
    t = Tables(1, 16, 60, 5, 12)
    for _ in range(35):
        t.kv.reserve(t.lens, t.table, t.free, t.n_free)
        t.m.reserve([1] * 5)
    t.kv.synchronize()
    assert t.same()


def test_lengths_and_number_to_other_arrays(gpu):
    t = Tables(2, 16, 60, 3, 12)
    t.reserve([20, 0, 5])
    t.m.reserve([20, 0, 5])
    before, free = t.lens.clone(), t.n_free.clone()
    lens_out, n_free_out = torch.zeros_like(t.lens), torch.zeros_like(t.n_free)
    for _ in range(2):  # the same twice
        slots = t.reserve([1, 17, 12], lens_out=lens_out, n_free_out=n_free_out)
        assert torch.equal(t.lens, before) and torch.equal(t.n_free, free)
    starts, want = t.m.reserve([1, 17, 12])
    t.lens, t.n_free = lens_out, n_free_out
    t.kv.synchronize()
    assert t.same() and slots.tolist() == want and t.starts.tolist() == starts


@pytest.mark.parametrize("seqs", [3, 100])
@pytest.mark.parametrize("what", ["too few pages", "table too short", "length below zero", "count below zero", "too few slots", "n_free below zero",
                                  "n_free beyond the pool", "sums beyond 2^31"])
def test_all_get_their_pages_or_none(gpu, seqs, what):
    page, wide = (256, 1 << 17) if what == "sums beyond 2^31" else (16, 10)
    t = Tables(3, page, 4 * seqs, seqs, wide)
    t.reserve([20] * seqs)
    new, n_rows = [3] * seqs, 3 * seqs
    lens, n_free = t.lens.clone(), t.n_free.clone()
    if what == "too few pages":
        new = [50] * seqs
        n_rows = 50 * seqs
    elif what == "table too short":
        new[seqs - 1] = 141
        n_rows += 200
    elif what == "length below zero":
        lens[seqs // 2] = -1
    elif what == "count below zero":
        new[seqs // 2] = -1
    elif what == "too few slots":
        n_rows -= 1
    elif what == "n_free below zero":
        n_free[0] = -1
    elif what == "n_free beyond the pool":
        n_free[0] = 4 * seqs + 1
    else:
        new = [(1 << 25) - 25] * seqs if seqs == 100 else [2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1]
    t.lens.copy_(lens), t.n_free.copy_(n_free)
    table, free = t.table.clone(), t.free.clone()
    slots = t.reserve(new, n_rows)
    with pytest.raises(U.UadError) as e:
        t.kv.synchronize()
    assert e.value.status == 9
    assert torch.equal(t.table, table) and torch.equal(t.free, free) and torch.equal(t.lens, lens) and torch.equal(t.n_free, n_free)
    assert bool((slots == -1).all()) and not bool(t.starts.any())


def test_the_last_page_can_be_taken(gpu):
    t = Tables(4, 16, 6, 2, 3)
    t.reserve([48, 48])
    t.kv.synchronize()
    assert t.m.reserve([48, 48]) and t.same() and t.n_free.tolist() == [0]
    t.reserve([0, 0])
    t.kv.synchronize()


def test_ids_outside_the_pool_give_no_slots(gpu):
    t = Tables(5, 16, 9, 2, 4)
    t.free[7] = 1 << 30
    slots = t.reserve([16, 20])
    with pytest.raises(U.UadError):
        t.kv.synchronize()
    got = slots.tolist()
    assert got[16:32] == [-1] * 16 and min(got[:16] + got[32:]) >= 0 and t.table[1].tolist()[0] == 1 << 30
    t.table[0, 0] = 1 << 30  # of a page that is begun
    t.lens[0] = 3
    slots = t.reserve([2, 0])
    with pytest.raises(U.UadError):
        t.kv.synchronize()
    assert slots.tolist() == [-1, -1]


@pytest.mark.parametrize("what", ["too many", "n_free below zero", "n_free beyond the pool", "an id beyond the pool", "length below zero"])
def test_release_reports_what_it_cannot_use(gpu, what):
    t = Tables(6, 16, 30, 3, 8)
    t.reserve([100, 20, 33])
    t.kv.synchronize()
    n_free = t.n_free.clone()
    t.lens.zero_()
    if what == "too many":
        t.n_free[0] = 28
    elif what == "n_free below zero":
        t.n_free[0] = -1
    elif what == "n_free beyond the pool":
        t.n_free[0] = 31
    elif what == "an id beyond the pool":
        t.table[1, 1] = 30
    else:
        t.lens[1] = -4
    table, given, free = t.table.clone(), t.n_free.clone(), t.free.clone()
    t.kv.release(t.lens, t.table, t.free, t.n_free)
    with pytest.raises(U.UadError) as e:
        t.kv.synchronize()
    assert e.value.status == 9
    if what == "an id beyond the pool":
        assert t.table[1].tolist() == [-1, 30] + [-1] * 6 and t.n_free.tolist() == [29] and bool((t.table[[0, 2]] == -1).all())
    elif what == "length below zero":
        assert torch.equal(t.table[1], table[1]) and t.n_free.tolist() == [28] and bool((t.table[[0, 2]] == -1).all())
    else:
        assert torch.equal(t.table, table) and torch.equal(t.n_free, given) and torch.equal(t.free, free)
    assert what != "too many" or n_free.tolist() == [18]


@pytest.mark.parametrize("cache", [BF16, "blocks"])
def test_a_run_of_them_together(gpu, cache):
    """Two conversations: pages for their prompts, the prompts appended and attended, then tokens by a captured step that
    takes pages, appends, attends with a window and sinks and gives pages back; then one goes and another comes in its
    pages.  Outputs against their definition over the tokens as the cache holds them."""
    hkv, heads, hd, page, n_pages, window, sinks, wide = 2, 6, 64, 16, 24, 40, 5, 12
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        kv = U.PagedKV(1, heads, hkv, hd, page, n_pages, 2, dtype=F8 if cache == "blocks" else BF16, rope_dim=hd, block_scales=cache == "blocks", stream=st)
        for t in (kv.k, kv.v) + ((kv.k_scales, kv.v_scales) if cache == "blocks" else ()):
            t.fill_(float("nan"))
        table = torch.full((2, wide), -1, dtype=I32, device="cuda")
        lens, n_free = torch.zeros(2, dtype=I32, device="cuda"), torch.tensor([n_pages], dtype=I32, device="cuda")
        free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(3)).to(I32).cuda()

        held = R.Cache(0, 1, hkv, hd, page, [1, 1], blocks=cache == "blocks", spare=n_pages)

        def attended(q, out, new, w, s):
            """`out` against the definition over what the pools hold now."""
            held.k, held.v, held.table, held.lens = kv.k.cpu(), kv.v.cpu(), table.cpu().numpy(), lens.cpu().numpy()
            if cache == "blocks":
                held.block = [kv.k_scales.cpu(), kv.v_scales.cpu()]
            want = R.attend_rows(held, 0, q.double().cpu().numpy(), new, hd, False, 1 / math.sqrt(hd), w, s)
            o, b, a, n = want
            assert np.all(np.abs(out.double().cpu().numpy() - o) <= R.rows_bound(o, b, n, hd, a, 2, BF16))

        def prompt(new):
            starts, slots = torch.zeros(3, dtype=I32, device="cuda"), torch.zeros(sum(new), dtype=torch.int64, device="cuda")
            q, k, v = (dev(draw(sum(new) + i, sum(new), h, hd)).to(BF16) for i, h in ((0, heads), (1, hkv), (2, hkv)))
            kv.reserve(lens, table, free, n_free, dev(np.array(new, np.int32)), starts, slots)
            kv.append(0, k, v, table, lens, starts)
            out = kv.attend_rows(0, q, table, lens, starts)
            kv.synchronize()
            # what went to the slots is what was appended
            flat = kv.v[0].permute(0, 3, 1, 2).reshape(-1, hkv, hd).float()[slots]
            if cache == "blocks":
                flat = flat * kv.v_scales[0].permute(0, 2, 1).reshape(-1, hkv)[slots // 16][..., None]
            assert float((flat - v.float()).abs().max()) <= (2.0 ** -4 * 6 if cache == "blocks" else 0)
            attended(q, out, new, 0, 0)

        prompt([50, 17])
        q, k, v = (torch.zeros((2, h, hd), dtype=BF16, device="cuda") for h in (heads, hkv, hkv))
        out = torch.zeros_like(q)

        def step():
            kv.reserve(lens, table, free, n_free)
            kv.append(0, k, v, table, lens)
            kv.attend_rows(0, q, table, lens, out=out, window=window, sinks=sinks)
            kv.release(lens, table, free, n_free, window, sinks)

        state = [t.clone() for t in (lens, table, free, n_free)]
        step()
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step()
        for t, s in zip((lens, table, free, n_free), state):
            t.copy_(s)
        for i in range(60):
            for x, s in ((q, 1), (k, 2), (v, 3)):
                x.copy_(draw(1000 * s + i, *x.shape))
            graph.replay()
            kv.synchronize()
            if i % 7 == 0 or i > 56:
                attended(q, out, [1, 1], window, sinks)
            used = int((table >= 0).sum())
            assert used + int(n_free) == n_pages and int(lens[0]) == 51 + i
        assert int((table[0] >= 0).sum()) <= 5  # the window's and the sinks'
        lens[0] = 0
        kv.release(lens, table, free, n_free, window, sinks)
        prompt([33, 0])
        kv.synchronize()
        ids = table[table >= 0].tolist()
        assert len(set(ids)) == len(ids) and sorted(ids + free[:int(n_free)].tolist()) == list(range(n_pages))


def test_calls_from_another_stream(gpu):
    """Page tables of a handle on a stream of its own, called from the default one."""
    st = torch.cuda.Stream()
    t = Tables(7, 16, 4000, 8, 300)
    kv = U.PagedKV(1, 1, 1, 64, 16, 4000, 8, dtype=F8, stream=st)
    t.kv = kv
    torch.cuda.synchronize()
    for i in range(20):
        new = [(i * 7 + b) % 40 for b in range(8)]
        keep = t.reserve(new)
        t.m.reserve(new)
        del keep  # its memory stays until the handle's stream is done
        kv.release(t.lens, t.table, t.free, t.n_free, 60, 3)
        t.m.release(60, 3)
    kv.synchronize()
    assert t.same()
