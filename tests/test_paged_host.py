"""The paged cache without a GPU: index arithmetic and device-side checks (csrc/paged.h compiled by the host compiler),
and the C ABI's refusals against a stand-in for the HIP runtime."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2609_37772_amd as U

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_37772_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
OK, INVALID, SHAPE, HIP, UNSUPPORTED, PAGE = 0, 1, 2, 5, 7, 9

SRC = r"""
#include "%s/paged.h"
using namespace uad;
extern "C" {
unsigned long long k_at(int np, int sh, int hkv, int hd, int page, int h, int off, int c) {
  PagedDims d{np, sh, hkv, hd}; return page_base(d, page, h) + k_in_page(d, off, c); }
unsigned long long v_at(int np, int sh, int hkv, int hd, int page, int h, int off, int c) {
  PagedDims d{np, sh, hkv, hd}; return page_base(d, page, h) + v_in_page(d, off, c); }
int ok(int np, int page) { PagedDims d{np, 4, 1, 64}; return page_ok(d, page); }
int usable(int len, int pages, int sh, int *bad) { bool b = false; int n = usable_length(len, pages, sh, &b); *bad = b; return n; }
void pair(int p, int rd, int nb, int *a, int *b) { rope_pair(p, rd, nb != 0, a, b); }
}
"""


@pytest.fixture(scope="module")
def idx(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged")
    src = d / "p.cpp"
    src.write_text(SRC % CSRC)
    subprocess.run(["g++", "-O1", "-Wall", "-Werror", "-std=c++17", "-shared", "-fPIC", "-Xlinker", "-z", "-Xlinker", "defs",
                    str(src), "-o", str(d / "p.so")], check=True)
    lib = ctypes.CDLL(str(d / "p.so"))
    lib.k_at.restype = lib.v_at.restype = ctypes.c_ulonglong
    return lib


@pytest.mark.parametrize("pages,shift,hkv,hd", [(3, 4, 1, 64), (2, 5, 3, 128), (70000, 8, 8, 256)])
def test_every_token_has_its_slot(idx, pages, shift, hkv, hd):
    ps = 1 << shift
    k = lambda p, h, o, c: ((p * hkv + h) * ps + o) * hd + c  # noqa: E731  [page][head][token][dim]
    v = lambda p, h, o, c: ((p * hkv + h) * hd + c) * ps + o  # noqa: E731  [page][head][dim][token]
    for p in (0, 1, pages - 1):
        for h in {0, hkv - 1}:
            for o in (0, 1, ps - 1):
                for c in (0, 8, hd - 1):
                    assert idx.k_at(pages, shift, hkv, hd, p, h, o, c) == k(p, h, o, c)
                    assert idx.v_at(pages, shift, hkv, hd, p, h, o, c) == v(p, h, o, c)
    assert pages < 70000 or k(pages - 1, hkv - 1, ps - 1, hd - 1) > 2 ** 35


def test_page_ids(idx):
    for n in (1, 5, 2 ** 31 - 1):
        assert [idx.ok(n, p) for p in (0, n - 1, -1, -2 ** 31)] == [1, 1, 0, 0]
        assert n == 2 ** 31 - 1 or not idx.ok(n, n)


@pytest.mark.parametrize("length,pages,shift,want,bad", [
    (0, 1, 4, 0, 0), (16, 1, 4, 16, 0), (17, 1, 4, 16, 1), (-1, 1, 4, 0, 1), (-2 ** 31, 9, 4, 0, 1), (2 ** 31 - 1, 1, 8, 256, 1),
    (2 ** 31 - 1, 2 ** 31 - 1, 8, 2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 23, 8, 2 ** 31 - 1, 0)])
def test_lengths(idx, length, pages, shift, want, bad):
    b = ctypes.c_int()
    assert idx.usable(length, pages, shift, ctypes.byref(b)) == want and b.value == bad


@pytest.mark.parametrize("hd,rd,nb", [(64, 64, 0), (64, 32, 0), (64, 32, 1), (128, 0, 0), (256, 256, 1), (128, 16, 0)])
def test_rotation_pairs_cover_a_head_once(idx, hd, rd, nb):
    seen = []
    for p in range(hd // 2):
        a, b = ctypes.c_int(), ctypes.c_int()
        idx.pair(p, rd, nb, ctypes.byref(a), ctypes.byref(b))
        seen += [a.value, b.value]
        if p < rd // 2:
            assert (a.value, b.value) == ((2 * p, 2 * p + 1) if nb else (p, p + rd // 2))
        else:
            assert a.value >= rd
    assert sorted(seen) == list(range(hd))


# ------------------------------------------------------------------------------------------------ the C ABI
@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("kvstub"))
    srcs = [os.path.join(CSRC, p) for p in ("uad_api.cpp", "kv_api.cpp", "schedule.cpp")]
    srcs += [os.path.join(ROOT, "tests", "stub", p) for p in ("hip_stub.cpp", "kv_stub.cpp")]
    objs = []
    for src in srcs:
        objs.append(os.path.join(d, os.path.basename(src) + ".o"))
        # the stand-in notes which device is current: its hipSetDevice takes the place of the other's
        more = ["-DhipSetDevice=kv_set_device"] if src.endswith("kv_api.cpp") else []
        more += ["-include", os.path.join(d, "decl.h")] if more else []
        if more:
            with open(os.path.join(d, "decl.h"), "w") as f:
                f.write("#include <hip/hip_runtime.h>\nextern \"C\" hipError_t kv_set_device(int);\n")
        subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-fPIC", "-std=c++17",
                        *more, "-c", src, "-o", objs[-1]], check=True)
    names = subprocess.run(["nm", "-u", *objs], capture_output=True, text=True, check=True).stdout.split()
    fat = ["-Wl,--defsym,%s=0" % n for n in names if n.startswith("__hip_fatbin")]
    so = os.path.join(d, "libkvstub.so")
    subprocess.run(["g++", "-shared", "-o", so, *objs, "-Wl,-z,defs", "-Wl,-Bsymbolic", *fat], check=True)
    lib = ctypes.CDLL(so)
    lib.kv_stub_calls.restype = lib.uad_kv_last_error.restype = lib.uad_last_error.restype = ctypes.c_char_p
    lib.uad_kv_attend.argtypes = U.load_library().uad_kv_attend.argtypes
    lib.uad_kv_append.argtypes = U.load_library().uad_kv_append.argtypes
    lib.uad_set_prefix_paged.argtypes = U.load_library().uad_set_prefix_paged.argtypes
    lib.stub_map.argtypes = [ctypes.c_void_p, ctypes.c_size_t]
    return lib


class Pools:
    def __init__(self, lib, elems, esz=2, short=0):
        self.lib = lib
        self.a = [np.zeros(elems * esz + 64, np.uint8) for _ in range(2)]
        self.p = [(a.ctypes.data + 15) // 16 * 16 for a in self.a]
        for i, p in enumerate(self.p):
            lib.stub_map(p, elems * esz - (short if i else 0))

    def close(self):
        for p in self.p:
            self.lib.stub_map(p, 0)


def config(pools, **kw):
    base = dict(n_layers=2, n_heads=4, n_kv_heads=2, head_dim=64, page_size=16, n_pages=3, max_seqs=4, dtype=1, rope_dim=64,
                rope_pairs=0, rope_theta=1e4, k_scale=1.0, v_scale=1.0, k=pools.p[0], v=pools.p[1])
    base.update(kw)
    return U._binding.uad_kv_config(**base)


ELEMS = 2 * 3 * 2 * 16 * 64


def create(lib, cfg):
    h = ctypes.c_void_p(99)
    return lib.uad_kv_create(ctypes.byref(cfg), 0, None, ctypes.byref(h)), h


@pytest.fixture
def kv(lib):
    pools = Pools(lib, ELEMS)
    st, h = create(lib, config(pools))
    assert st == OK
    lib.kv_stub_reset(0)
    yield h
    lib.uad_kv_destroy(h)
    pools.close()


@pytest.mark.parametrize("change,status", [
    (dict(n_layers=0), INVALID), (dict(n_heads=-1), INVALID), (dict(n_kv_heads=0), INVALID), (dict(head_dim=0), INVALID),
    (dict(page_size=0), INVALID), (dict(n_pages=0), INVALID), (dict(max_seqs=0), INVALID), (dict(dtype=0), INVALID),
    (dict(dtype=3), INVALID), (dict(rope_dim=-16), INVALID), (dict(rope_dim=80), INVALID), (dict(rope_pairs=2), INVALID),
    (dict(rope_theta=0.0), INVALID), (dict(rope_theta=float("nan")), INVALID), (dict(rope_theta=float("inf")), INVALID),
    (dict(dtype=2, k_scale=0.0), INVALID), (dict(dtype=2, v_scale=float("inf")), INVALID), (dict(dtype=2, k_scale=-1.0), INVALID),
    (dict(dtype=2, k_scale=1e-45), INVALID), (dict(k_scale=2.0), INVALID), (dict(v_scale=0.5), INVALID),
    (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=512), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED),
    (dict(page_size=48), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED), (dict(rope_dim=24), UNSUPPORTED),
    (dict(n_heads=3), UNSUPPORTED), (dict(n_heads=2 ** 26), UNSUPPORTED), (dict(max_seqs=2 ** 22), UNSUPPORTED), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(n_pages=4), SHAPE), (dict(n_layers=3), SHAPE), (dict(n_pages=2 ** 31 - 1, n_layers=2 ** 31 - 1), SHAPE),
])
def test_create_refuses(lib, change, status):
    pools = Pools(lib, ELEMS)
    st, h = create(lib, config(pools, **change))
    assert st == status and h.value is None
    assert lib.uad_kv_last_error(None).startswith(b"uad_kv_create: ")
    pools.close()


def test_create_refuses_pools_that_are_unaligned_short_or_host_memory(lib):
    pools = Pools(lib, ELEMS)
    assert create(lib, config(pools, k=pools.p[0] + 8))[0] == INVALID
    pools.close()
    assert create(lib, config(pools))[0] == SHAPE  # no longer device memory
    pools = Pools(lib, ELEMS, short=1)
    assert create(lib, config(pools))[0] == SHAPE
    pools.close()
    pools = Pools(lib, ELEMS, esz=1)  # enough for 8 bits only
    assert create(lib, config(pools))[0] == SHAPE
    st, h = create(lib, config(pools, dtype=2, k_scale=0.5))
    assert st == OK
    lib.uad_kv_destroy(h)
    pools.close()
    assert lib.uad_kv_create(None, 0, None, None) == INVALID
    lib.uad_kv_destroy(None)


X = 0x7f0000001000  # an address that host code never reads


def append(lib, h, **kw):
    a = dict(layer=0, k=X, v=X, dtype=1, ldk=128, ldv=128, n_rows=3, row_start=X, lens=X, positions=None, table=X, pages=2, n_seqs=2)
    a.update(kw)
    return lib.uad_kv_append(h, *a.values())


def attend(lib, h, **kw):
    a = dict(layer=0, q=X, out=X, dtype=1, ldq=256, ldo=256, lens=X, positions=None, table=X, pages=2, n_seqs=2, scale=1.0)
    a.update(kw)
    return lib.uad_kv_attend(h, *a.values())


@pytest.mark.parametrize("change,status", [
    (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID),
    (dict(pages=0), INVALID), (dict(n_seqs=-1), INVALID), (dict(n_seqs=5), SHAPE), (dict(lens=None), INVALID),
    (dict(table=None), INVALID), (dict(pages=2 ** 26 + 1), SHAPE), (dict(pages=2 ** 31 - 1), SHAPE)])
def test_calls_refuse_alike(lib, kv, change, status):
    for call in (append, attend):
        assert call(lib, kv, **change) == status
        assert lib.uad_kv_last_error(kv).startswith(b"uad_kv_")
    assert lib.kv_stub_calls() == b""


@pytest.mark.parametrize("change,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ldk=127), INVALID), (dict(ldv=0), INVALID), (dict(n_rows=-1), INVALID),
    (dict(ldk=2 ** 30 + 1), INVALID), (dict(ldv=2 ** 62), INVALID), (dict(row_start=None), SHAPE), (dict(k=X + 1), INVALID), (dict(dtype=0, v=X + 2), INVALID)])
def test_append_refuses(lib, kv, change, status):
    assert append(lib, kv, **change) == status and lib.kv_stub_calls() == b""


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(ldq=255), INVALID), (dict(ldo=-256), INVALID),
    (dict(ldq=2 ** 30 + 1), INVALID), (dict(scale=3e38), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(q=X + 1), INVALID), (dict(dtype=0, out=X + 2), INVALID)])
def test_attend_refuses(lib, kv, change, status):
    assert attend(lib, kv, **change) == status and lib.kv_stub_calls() == b""


def test_calls_go_through_and_leave_the_callers_device(lib, kv):
    before = lib.kv_stub_current_device()
    assert before == 3  # the handle's device is 0
    assert append(lib, kv) == OK and append(lib, kv, n_rows=2, row_start=None, dtype=0, ldk=999) == OK and attend(lib, kv) == OK
    assert lib.kv_stub_calls() == b"append 3 2 0 0 128 128 4;append 2 2 1 0 999 128 4;attend 2 4 2 0 0;"
    assert lib.kv_stub_current_device() == before
    lib.kv_stub_reset(0)
    # nothing to do: nothing is launched, and no pointer is needed
    assert append(lib, kv, n_rows=0, k=None, v=None) == OK and append(lib, kv, n_seqs=0, n_rows=0, row_start=None, lens=None, table=None) == OK
    assert attend(lib, kv, n_seqs=0, q=None, out=None, lens=None, table=None) == OK
    assert lib.kv_stub_calls() == b""
    lib.kv_stub_reset(1)
    assert append(lib, kv) == HIP and b"stub error" in lib.uad_kv_last_error(kv) and attend(lib, kv) == HIP
    assert lib.uad_kv_append(None, *[0] * 13) == INVALID and lib.uad_kv_synchronize(None) == INVALID


def test_status_word_is_reported_once(lib, kv):
    assert lib.uad_kv_synchronize(kv) == OK
    lib.kv_stub_status(kv, 4)
    assert lib.uad_kv_synchronize(kv) == PAGE and lib.uad_kv_last_error(kv)
    assert lib.uad_kv_synchronize(kv) == OK


@pytest.fixture
def ctx(lib):
    cfg = U._binding.uad_model_config(2, 128, 4, 2, 64, 256, 7, 2, 8, 40, 1e-6, 0)
    c = ctypes.c_void_p()
    assert lib.uad_create(ctypes.byref(cfg), 0, None, ctypes.byref(c)) == OK
    yield c
    lib.uad_destroy(c)


def test_prefix_from_pages(lib, kv, ctx):
    call = lambda **kw: lib.uad_set_prefix_paged(*{**dict(c=ctx, kv=kv, lens=X, table=X, pages=3, batch=2, n=40), **kw}.values())  # noqa: E731
    for change, status in ((dict(kv=None), INVALID), (dict(lens=None), INVALID), (dict(table=None), INVALID), (dict(batch=0), INVALID),
                           (dict(n=-1), INVALID), (dict(pages=0), INVALID), (dict(batch=3), SHAPE), (dict(n=41), SHAPE),
                           (dict(pages=2), SHAPE), (dict(c=None), INVALID)):
        assert call(**change) == status
    assert lib.kv_stub_calls() == b"" and lib.kv_stub_prefix_set(ctx) == -1
    assert call() == OK and lib.kv_stub_calls() == b"prefix 2 2 40;" and lib.kv_stub_prefix_set(ctx) == 40
    assert call(n=0) == OK and lib.kv_stub_prefix_set(ctx) == 0
    lib.kv_stub_reset(1)
    assert call() == HIP and lib.kv_stub_prefix_set(ctx) == -1  # an error leaves no prefix
    lib.kv_stub_reset(0)
    lib.kv_stub_ctx_status(ctx, 4)
    assert lib.uad_synchronize(ctx) == PAGE and lib.uad_synchronize(ctx) == OK


@pytest.mark.parametrize("change", [dict(n_layers=1), dict(n_kv_heads=1), dict(head_dim=128, n_pages=1)])
def test_prefix_from_another_models_pages_is_refused(lib, ctx, change):
    pools = Pools(lib, ELEMS)
    st, h = create(lib, config(pools, **change))
    assert st == OK
    lib.kv_stub_reset(0)
    assert lib.uad_set_prefix_paged(ctx, h, X, X, 3, 2, 16) == SHAPE and lib.kv_stub_calls() == b""
    lib.uad_kv_destroy(h)
    pools.close()


# ------------------------------------------------------------------------------------------------ the attention's plan
PLAN = r"""
#include "%s/paged.h"
using namespace uad;
extern "C" {
int tiles_of(int len, int tile) { return tiles_of_length(len, tile); }
int share_of(long long total, int target, int least) { return first_share(total, target, least); }
int larger(int share) { return next_share(share); }
int splits(int tiles, int share, int whole) { return splits_of(tiles, share, whole); }
int begin(int tiles, int n, int s) { return split_begin(tiles, n, s); }
int slots(int target) { return max_slots(target); }
int tries() { return kShareTries; }
int fan() { return kJoinFan; }
int most() { return kMaxSplits; }
int tile_shift(int page_shift) { return append_tile_shift(page_shift); }
int append_tiles_of(int from, int to, int shift) { return append_tiles(from, to, shift); }
long long append_wgs(int rows, int seqs, int shift) { return append_grid(rows, seqs, shift); }
int rows_fine(int from, int to, int rows) { return rows_ok(from, to, rows); }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "p.cpp").write_text(PLAN % CSRC)
    subprocess.run(["g++", "-O1", "-Wall", "-Werror", "-std=c++17", "-shared", "-fPIC", str(d / "p.cpp"), "-o", str(d / "p.so")], check=True)
    lib = ctypes.CDLL(str(d / "p.so"))
    lib.append_wgs.restype = ctypes.c_longlong
    lib.share_of.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    return lib


def plan_of(lib, lens, units, tile, target, least=4, whole=4):
    tiles = [lib.tiles_of(n, tile) for n in lens]
    total = sum(tiles) * units
    share = lib.share_of(total, target, least)
    count = lambda: sum(lib.splits(t, share, whole) * units for t in tiles)  # noqa: E731
    if len(lens) * units < target:
        for _ in range(lib.tries()):
            if count() <= target:
                break
            share = lib.larger(share)
    return tiles, share, [lib.splits(t, share, whole) for t in tiles]


def test_plan_covers_every_tile_within_the_slots_and_the_grid(plan):
    r = np.random.default_rng(3)
    for _ in range(400):
        n, units, target = int(2 ** r.uniform(0, 8)), int(2 ** r.uniform(0, 5)), int(r.choice([1, 64, 256, 304, 512, 768]))
        tile, pages, shift = int(r.choice([32, 64])), int(2 ** r.uniform(0, 14)), int(r.integers(4, 9))
        cap = min(pages << shift, 2 ** 31 - 1)
        lens = [int(x) for x in np.minimum(2 ** r.uniform(0, r.choice([3, 12, 22, 31]), n) - 1, cap)]
        whole = int(r.choice([1, 4, 8, 12, 20]))
        tiles, share, splits = plan_of(plan, lens, units, tile, target, whole=whole)
        wgs, slots = sum(splits) * units, sum(s * units for s in splits if s > 1)
        assert slots <= plan.slots(target) and max(splits) <= plan.most() and -(-max(splits) // plan.fan()) <= 2 * plan.fan()
        # the launch: as many workgroups as the lengths could need
        most = plan.splits(plan.tiles_of(cap, tile), 4, whole)
        assert wgs <= min(n * units * most, n * units + plan.slots(target))
        for t, s in zip(tiles, splits):
            ends = [plan.begin(t, s, i) for i in range(s + 1)]
            assert ends[0] == 0 and ends[-1] == t and all(b > a for a, b in zip(ends, ends[1:]))
            assert s == plan.most() or max(b - a for a, b in zip(ends, ends[1:])) <= max(share, whole)
            assert t > whole or s == 1


def test_plan_fills_the_workgroups_that_run_at_once(plan):
    for n, units, length in ((1, 1, 817), (64, 1, 900), (1, 8, 131071), (8, 16, 4001), (1, 1, 1 << 20)):
        tiles, share, splits = plan_of(plan, [length] * n, units, 32, 256)
        wgs = sum(splits) * units
        assert wgs <= 256 and (wgs >= 200 or share == 4)
    assert plan_of(plan, [0], 4, 32, 256)[2] == [1]


def test_append_tiles_hold_every_row_once_within_the_grid(plan):
    r = np.random.default_rng(4)
    for _ in range(400):
        page_shift = int(r.integers(4, 9))
        shift = plan.tile_shift(page_shift)
        assert shift <= page_shift and 1 << shift <= 64
        n = int(2 ** r.uniform(0, 8))
        new = (2 ** r.uniform(0, r.choice([1, 4, 11]), n) - 1 + r.integers(0, 2)).astype(int)
        before = r.integers(0, 300, n)
        total = 0
        for a, b in zip(before, before + new):
            tiles = {p >> shift for p in range(a, b)}
            assert plan.append_tiles_of(int(a), int(b), shift) == len(tiles)
            total += len(tiles)
        if new.sum():
            assert total <= plan.append_wgs(int(new.sum()), n, shift)
    assert [plan.rows_fine(*x) for x in ((0, 0, 0), (0, 5, 5), (2, 1, 9), (-1, 2, 9), (3, 10, 9))] == [1, 1, 0, 0, 0]
