"""New rows' attention, scales for blocks and page tables without a GPU: index arithmetic (csrc/paged.h compiled by the host
compiler), the C ABI's refusals against a stand-in for the HIP runtime, and the binding's."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
from tests import rows_oracle as R
from tests.test_paged_host import CSRC, ELEMS, HIP, HIPCC, INVALID, OK, ROOT, SHAPE, UNSUPPORTED, Pools, config

SRC = r"""
#include "%s/paged.h"
using namespace uad;
extern "C" {
unsigned long long scale_at(int np, int sh, int hkv, int hd, int page, int h, int off) { PagedDims d{np, sh, hkv, hd}; return scale_index(d, page, h, off); }
unsigned bits_of_scale(unsigned most) { return scale_bits(most); }
int from(int p, int w) { return seen_from(p, w); }
int to(int p, int len, int w, int causal) { return seen_to(p, len, w, causal != 0); }
int first(int p, int len, int s, int causal) { return seen_first(p, len, s, causal != 0); }
void tiles(int len, int lo, int sinks, int tile, int *o) { SeenTiles s = seen_tiles(len, lo, sinks, tile); o[0] = s.first; o[1] = s.gap; o[2] = s.count; }
int tile_of(int first, int gap, int i) { SeenTiles s{first, gap, 0}; return seen_tile(s, i); }
unsigned run(int from, int to, int n) { return run_bits(from, to, n); }
int pages(int len, int shift) { return pages_of(len, shift); }
int grows(int len, int n, int pages, int shift) { return growth_ok(len, n, pages, shift); }
unsigned long long steps(double turns) { return steps_of(turns); }
int used(int i, int len, int w, int s, int shift) { return page_in_use(i, len, w, s, shift); }
}
"""


@pytest.fixture(scope="module")
def idx(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    (d / "p.cpp").write_text(SRC % CSRC)
    subprocess.run(["g++", "-O1", "-Wall", "-Werror", "-std=c++17", "-shared", "-fPIC", str(d / "p.cpp"), "-o", str(d / "p.so")], check=True)
    lib = ctypes.CDLL(str(d / "p.so"))
    lib.scale_at.restype = ctypes.c_ulonglong
    lib.bits_of_scale.restype = lib.run.restype = ctypes.c_uint
    lib.bits_of_scale.argtypes = [ctypes.c_uint]
    return lib


def test_turns_in_whole_numbers(idx):
    idx.steps.restype, idx.steps.argtypes = ctypes.c_ulonglong, [ctypes.c_double]
    r = np.random.default_rng(5)
    from fractions import Fraction
    for x in [0.0, 0.15915494309189535, 1 - 2.0 ** -53, 1.0, 2.0 ** -70, 1234567.75, 2.0 ** 53, 1e300] + list(10.0 ** r.uniform(-9, 3, 200)):
        want = int((Fraction(float(x)) % 1) * 2 ** 64)
        assert abs(idx.steps(x) - want) <= 1, x


def test_every_block_has_its_scale(idx):
    for pages, shift, hkv in ((3, 4, 2), (5, 6, 1), (70000, 8, 300)):
        per = (1 << shift) // 16
        for p in (0, 1, pages - 1):
            for h in {0, hkv - 1}:
                for off in {0, 15, (1 << shift) - 1}:
                    assert idx.scale_at(pages, shift, hkv, 64, p, h, off) == (p * hkv + h) * per + off // 16


def test_scales_are_the_least_powers_of_two(idx):
    scale = lambda x: float(np.uint32(idx.bits_of_scale(int(np.float32(x).view(np.uint32)))).view(np.float32))  # noqa: E731
    edge = [np.float32(448 * 2.0 ** e) for e in (-110, -100, -7, 0, 1, 60, 119)]
    values = [0.0, 1e-45, 1.0, 3.4028235e38, 447.0, 449.0] + edge
    values += [np.nextafter(x, np.float32(s)) for x in edge for s in (0, np.inf) if np.isfinite(np.nextafter(x, np.float32(s)))]
    values += list(np.float32(2.0) ** np.random.default_rng(1).uniform(-126, 127, 300).astype(np.float32))
    for x in values:
        assert scale(x) == R.block_scale(float(x)), x
    assert scale(448.0) == 1.0 and scale(np.nextafter(np.float32(448), np.float32(999))) == 2.0


def test_rows_see_what_they_are_defined_to(idx):
    r = np.random.default_rng(2)
    for _ in range(300):
        m = int(r.integers(1, 80))
        n, w, s, causal = int(r.integers(1, m + 1)), int(r.integers(0, 90)), int(r.integers(0, 90)), int(r.integers(0, 2))
        s = s if w else 0
        want = R.sees(n, m, w, s, bool(causal))
        for j in range(n):
            p = m - n + j
            lo, hi = getattr(idx, "from")(p, w), idx.to(p, m, w, causal)
            got = [lo <= x < hi or x < idx.first(p, m, s, causal) for x in range(m)]
            assert got == list(want[j]), (m, n, w, s, causal, j)
    big = 2 ** 30
    assert getattr(idx, "from")(big - 1, big) == 0 and idx.to(big - 1, big, big, 0) == big and getattr(idx, "from")(5, big) == 0
    assert getattr(idx, "from")(-1, 1) == 0 and idx.to(0, 1, 2 ** 30, 0) == 1


def test_tiles_hold_every_key_that_is_seen(idx):
    r = np.random.default_rng(3)
    for _ in range(500):
        tile, m = int(r.choice([32, 64])), int(r.integers(0, 700))
        n = int(r.integers(1, max(2, m + 1)))
        w, s = int(r.integers(1, 300)), int(r.integers(0, 300))
        lo = getattr(idx, "from")(m - n, w)
        o = (ctypes.c_int * 3)()
        idx.tiles(m, lo, s, tile, o)
        first, gap, count = o
        assert first >= 0 and gap >= 0 and count >= 1
        at = [idx.tile_of(first, gap, i) for i in range(count)]
        assert at == sorted(set(at)) and (m == 0 or at[-1] == (m - 1) // tile)
        have = {t * tile + i for t in at for i in range(tile)}
        assert all(x in have for x in range(m) if x >= lo or x < s)
        assert count <= (w + n) // tile + s // tile + 4  # what the launch counts with
    o = (ctypes.c_int * 3)()
    idx.tiles(2 ** 30, 2 ** 30 - 5, 2 ** 30, 64, o)
    assert list(o) == [2 ** 24 - 1, 0, 2 ** 24]


def test_runs_of_keys_as_bits(idx):
    for n in (8, 16, 32):
        for a in range(-5, n + 6):
            for b in range(-5, n + 6):
                assert idx.run(a, b, n) == sum(1 << i for i in range(n) if a <= i < b)
    assert idx.run(-2 ** 30, 2 ** 30, 16) == 0xFFFF and idx.run(2 ** 30, 2 ** 30 + 1, 16) == 0


def test_pages_of_sequences(idx):
    for shift in (4, 8):
        p = 1 << shift
        assert [idx.pages(n, shift) for n in (0, 1, p, p + 1, 2 ** 30)] == [0, 1, 1, 2, 2 ** 30 // p]
        for len_, n, pages, want in ((0, 0, 1, 1), (0, p, 1, 1), (1, p, 1, 0), (-1, 1, 9, 0), (1, -1, 9, 0), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 22, 0)):
            assert idx.grows(len_, n, pages, shift) == want
        for m in (0, 1, p - 1, p, 3 * p + 5):
            for w, s in ((0, 0), (1, 0), (p, 0), (p + 1, 1), (5, p + 1), (2 ** 30, 2 ** 30)):
                for i in range(6):
                    want = any(x < s or w == 0 or x > m - w for x in range(i * p, min(m, (i + 1) * p))) or (m % p > 0 and i == m // p)
                    assert idx.used(i, m, w, s, shift) == want, (m, w, s, i)


# ------------------------------------------------------------------------------------------------ the C ABI
@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("kvrowsstub"))
    srcs = [os.path.join(CSRC, p) for p in ("uad_api.cpp", "kv_api.cpp", "kv_rows_api.cpp", "schedule.cpp")]
    srcs += [os.path.join(ROOT, "tests", "stub", p) for p in ("hip_stub.cpp", "kv_stub.cpp", "kv_rows_stub.cpp")]
    with open(os.path.join(d, "decl.h"), "w") as f:
        f.write("#include <hip/hip_runtime.h>\nextern \"C\" hipError_t kv_set_device(int);\n")
    objs = []
    for src in srcs:
        objs.append(os.path.join(d, os.path.basename(src) + ".o"))
        more = ["-DhipSetDevice=kv_set_device", "-include", os.path.join(d, "decl.h")] if "/kv_" in src and src.endswith("api.cpp") else []
        subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-fPIC", "-std=c++17",
                        *more, "-c", src, "-o", objs[-1]], check=True)
    names = subprocess.run(["nm", "-u", *objs], capture_output=True, text=True, check=True).stdout.split()
    fat = ["-Wl,--defsym,%s=0" % n for n in names if n.startswith("__hip_fatbin")]
    so = os.path.join(d, "libkvrowsstub.so")
    subprocess.run(["g++", "-shared", "-o", so, *objs, "-Wl,-z,defs", "-Wl,-Bsymbolic", *fat], check=True)
    lib, real = ctypes.CDLL(so), U.load_library()
    lib.kv_rows_stub_calls.restype = lib.uad_kv_last_error.restype = ctypes.c_char_p
    for name in ("uad_kv_attend_rows", "uad_kv_reserve", "uad_kv_release", "uad_kv_set_block_scales"):
        getattr(lib, name).argtypes = getattr(real, name).argtypes
    lib.stub_map.argtypes = [ctypes.c_void_p, ctypes.c_size_t]
    return lib


def made(lib, **kw):
    pools = Pools(lib, ELEMS)
    h = ctypes.c_void_p()
    assert lib.uad_kv_create(ctypes.byref(config(pools, **kw)), 0, None, ctypes.byref(h)) == OK
    lib.kv_rows_stub_reset(0)
    return pools, h


@pytest.fixture
def kv(lib):
    pools, h = made(lib)
    yield h
    lib.uad_kv_destroy(h)
    pools.close()


X = 0x7f0000001000  # an address that host code never reads


def rows(lib, h, **kw):
    a = dict(layer=0, q=X, out=X, dtype=1, ldq=256, ldo=256, n_rows=3, row_start=X, lens=X, positions=None, table=X, pages=2, n_seqs=2,
             scale=1.0, window=0, sinks=0, causal=1)
    a.update(kw)
    return lib.uad_kv_attend_rows(h, *a.values())


def reserve(lib, h, **kw):
    a = dict(lens=X, new=X, lens_out=X, table=X, pages=2, n_seqs=2, free=X, n_free=X, n_free_out=X, row_start=X, slots=X, n_rows=3)
    a.update(kw)
    return lib.uad_kv_reserve(h, *a.values())


def release(lib, h, **kw):
    a = dict(lens=X, table=X, pages=2, n_seqs=2, free=X, n_free=X, window=0, sinks=0)
    a.update(kw)
    return lib.uad_kv_release(h, *a.values())


@pytest.mark.parametrize("change,status", [
    (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(dtype=2), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID),
    (dict(ldq=255), INVALID), (dict(ldo=2 ** 30 + 1), INVALID), (dict(n_rows=-1), INVALID), (dict(row_start=None), SHAPE),
    (dict(lens=None), INVALID), (dict(table=None), INVALID), (dict(pages=0), INVALID), (dict(pages=2 ** 26 + 1), SHAPE), (dict(n_seqs=5), SHAPE),
    (dict(n_seqs=-1), INVALID), (dict(scale=float("nan")), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1, window=3), INVALID),
    (dict(sinks=1), INVALID), (dict(causal=2), INVALID), (dict(causal=-1), INVALID), (dict(q=X + 1), INVALID), (dict(dtype=0, out=X + 2), INVALID),
    (dict(n_rows=2 ** 23 + 1), SHAPE)])
def test_attend_rows_refuses(lib, kv, change, status):
    assert rows(lib, kv, **change) == status and lib.kv_rows_stub_calls() == b""
    assert lib.uad_kv_last_error(kv).startswith(b"uad_kv_attend_rows: ")


@pytest.mark.parametrize("change,status", [
    (dict(lens=None), INVALID), (dict(lens_out=None), INVALID), (dict(table=None), INVALID), (dict(free=None), INVALID), (dict(n_free=None), INVALID),
    (dict(n_free_out=None), INVALID), (dict(pages=0), INVALID), (dict(n_seqs=-1), INVALID), (dict(n_seqs=5), SHAPE), (dict(pages=2 ** 26 + 1), SHAPE),
    (dict(n_rows=-1), INVALID), (dict(slots=X + 4), INVALID)])
def test_reserve_refuses(lib, kv, change, status):
    assert reserve(lib, kv, **change) == status and lib.kv_rows_stub_calls() == b""
    assert lib.uad_kv_last_error(kv).startswith(b"uad_kv_reserve: ")


@pytest.mark.parametrize("change,status", [
    (dict(lens=None), INVALID), (dict(table=None), INVALID), (dict(free=None), INVALID), (dict(n_free=None), INVALID), (dict(pages=0), INVALID),
    (dict(n_seqs=5), SHAPE), (dict(window=-1), INVALID), (dict(window=4, sinks=-1), INVALID), (dict(sinks=4), INVALID)])
def test_release_refuses(lib, kv, change, status):
    assert release(lib, kv, **change) == status and lib.kv_rows_stub_calls() == b""
    assert lib.uad_kv_last_error(kv).startswith(b"uad_kv_release: ")


def test_calls_go_through_and_leave_the_callers_device(lib, kv):
    before = lib.kv_stub_current_device()
    assert rows(lib, kv) == rows(lib, kv, n_rows=2, row_start=None, dtype=0, window=2 ** 31 - 1, sinks=2 ** 31 - 1, causal=0, ldq=999) == OK
    assert reserve(lib, kv) == reserve(lib, kv, new=None, row_start=None, slots=None, n_rows=7) == release(lib, kv, window=9, sinks=1) == OK
    assert lib.kv_rows_stub_calls() == (b"rows 3 2 1 0 0 0 0 1 0;rows 2 2 0 1 0 1073741824 1073741824 0 0;reserve 2 3 1 3 4;reserve 2 0 0 3 4;"
                                        b"release 2 9 1 3;")
    assert lib.kv_stub_current_device() == before
    lib.kv_rows_stub_reset(0)
    # nothing to do: nothing is launched, and no pointer is needed
    assert rows(lib, kv, n_rows=0, q=None, out=None) == rows(lib, kv, n_rows=0, n_seqs=0, lens=None, table=None, row_start=None) == OK
    assert reserve(lib, kv, n_seqs=0, lens=None, table=None) == release(lib, kv, n_seqs=0, lens=None, table=None) == OK
    assert lib.kv_rows_stub_calls() == b""
    lib.kv_rows_stub_reset(1)
    for call in (rows, reserve, release):
        assert call(lib, kv) == HIP and b"stub error" in lib.uad_kv_last_error(kv)
    assert lib.uad_kv_attend_rows(None, *[0] * 17) == lib.uad_kv_reserve(None, *[0] * 12) == lib.uad_kv_release(None, *[0] * 8) == INVALID
    assert lib.uad_kv_set_block_scales(None, X, X) == INVALID


def test_block_scales_are_checked(lib):
    n = 2 * 3 * 2 * (16 // 16) * 4
    memory = np.zeros(2 * n + 64, np.uint8)
    at = (memory.ctypes.data + 15) // 16 * 16
    lib.stub_map(at, n)
    lib.stub_map(at + n, n)
    for kw, status in ((dict(), INVALID), (dict(dtype=2, k_scale=2.0), INVALID), (dict(dtype=2, v_scale=0.5), INVALID)):
        pools, h = made(lib, **kw)
        assert lib.uad_kv_set_block_scales(h, at, at + n) == status and not lib.kv_stub_has_scales(h)
        lib.uad_kv_destroy(h)
        pools.close()
    pools, h = made(lib, dtype=2)
    for k, v, status in ((at, None, INVALID), (None, at, INVALID), (at + 2, at + n, INVALID), (X, at, SHAPE), (at, at + n + 4, SHAPE)):
        assert lib.uad_kv_set_block_scales(h, k, v) == status and not lib.kv_stub_has_scales(h)
    assert lib.uad_kv_set_block_scales(h, at, at + n) == OK and lib.kv_stub_has_scales(h)
    assert rows(lib, h) == OK and lib.kv_rows_stub_calls().endswith(b" 1;")
    assert lib.uad_kv_set_block_scales(h, X, X) == SHAPE and lib.kv_stub_has_scales(h)  # an error leaves what was
    assert lib.uad_kv_set_block_scales(h, None, None) == OK and not lib.kv_stub_has_scales(h)
    lib.uad_kv_destroy(h)
    pools.close()
    lib.stub_map(at, 0)
    lib.stub_map(at + n, 0)
    big = 2 * 65536 * 16 * 64  # pools of one layer and page with more KV heads than a grid has rows
    spot = np.zeros(16, np.uint8).ctypes.data // 16 * 16 + 2 ** 40
    lib.stub_map(spot, big)
    h = ctypes.c_void_p()
    cfg = config(pools, dtype=2, n_layers=1, n_pages=1, n_heads=65536, n_kv_heads=65536, max_seqs=1, k=spot, v=spot)
    assert lib.uad_kv_create(ctypes.byref(cfg), 0, None, ctypes.byref(h)) == OK
    assert lib.uad_kv_set_block_scales(h, at, at) == UNSUPPORTED
    lib.uad_kv_destroy(h)
    lib.stub_map(spot, 0)


# ------------------------------------------------------------------------------------------------ the binding, on CPU tensors (device -1)
B, HQ, HD, DEV, I32 = U._binding, 4, 64, -1, torch.int32


@pytest.fixture
def calls(monkeypatch):
    seen, real = [], U.load_library()
    names = ("uad_kv_attend_rows", "uad_kv_reserve", "uad_kv_release")
    fns = {n: ctypes.CFUNCTYPE(ctypes.c_int32, *getattr(real, n).argtypes)(lambda *a, n=n: seen.append((n, *a)) or 0) for n in names}
    fake = type("Lib", (), {**{n: staticmethod(f) for n, f in fns.items()}, "uad_kv_last_error": staticmethod(lambda kv: b"")})
    monkeypatch.setattr(B, "load_library", lambda: fake)
    for n in ("_rows_at", "_reserve_at", "_release_at"):
        if hasattr(B, n):
            monkeypatch.setattr(B, n, ctypes.cast(fns["uad_kv_" + ("attend_rows" if n == "_rows_at" else n[1:-3])], ctypes.c_void_p).value)
    return seen


def ints(*shape):
    return torch.zeros(shape, dtype=I32)


def rows_call(**kw):
    x = torch.zeros((5, HQ, HD), dtype=torch.bfloat16)
    a = dict(kv=0x1234, layer=2, q=x, out=x.clone(), page_table=ints(3, 7), lens=ints(3), row_start=ints(4), positions=None, scale=0.5, window=9,
             n_sinks=2, causal=True, row_shape=(HQ, HD), device=DEV)
    a.update(kw)
    return a


def reserve_call(**kw):
    a = dict(kv=0x1234, lens=ints(3), page_table=ints(3, 7), free_pages=ints(9), n_free=ints(1), new_tokens=ints(3), row_start=ints(4),
             slots=torch.zeros(6, dtype=torch.int64), lens_out=ints(3), n_free_out=ints(1), n_pages=9, device=DEV)
    a.update(kw)
    return a


def release_call(**kw):
    a = dict(kv=0x1234, lens=ints(3), page_table=ints(3, 7), free_pages=ints(9), n_free=ints(1), window=5, n_sinks=1, n_pages=9, device=DEV)
    a.update(kw)
    return a


def test_the_binding_hands_over_what_it_is_given(calls):
    a = rows_call()
    B.uad_kv_attend_rows(**a)
    assert calls[-1] == ("uad_kv_attend_rows", 0x1234, 2, a["q"].data_ptr(), a["out"].data_ptr(), 1, 256, 256, 5, a["row_start"].data_ptr(),
                         a["lens"].data_ptr(), None, a["page_table"].data_ptr(), 7, 3, 0.5, 9, 2, 1)
    wide = torch.zeros((5, 3 * HQ, HD))
    a = rows_call(q=wide[:, HQ:2 * HQ], out=torch.zeros((5, HQ, HD)), positions=ints(5), causal=False, window=0, n_sinks=0, scale=2)
    B.uad_kv_attend_rows(**a)
    assert calls[-1][5:8] == (0, 3 * HQ * HD, HQ * HD) and calls[-1][11] == a["positions"].data_ptr() and calls[-1][15:] == (2.0, 0, 0, 0)
    a = rows_call(q=rows_call()["q"][:3], out=rows_call()["q"][:3], row_start=None)
    B.uad_kv_attend_rows(**a)
    assert calls[-1][8:10] == (3, None)
    a = reserve_call()
    B.uad_kv_reserve(**a)
    p = {k: v.data_ptr() for k, v in a.items() if isinstance(v, torch.Tensor)}
    assert calls[-1] == ("uad_kv_reserve", 0x1234, p["lens"], p["new_tokens"], p["lens_out"], p["page_table"], 7, 3, p["free_pages"], p["n_free"],
                         p["n_free_out"], p["row_start"], p["slots"], 6)
    B.uad_kv_reserve(**reserve_call(new_tokens=None, row_start=None, slots=None))
    assert calls[-1][3] is None and calls[-1][11:] == (None, None, 0)
    a = release_call()
    B.uad_kv_release(**a)
    assert calls[-1] == ("uad_kv_release", 0x1234, a["lens"].data_ptr(), a["page_table"].data_ptr(), 7, 3, a["free_pages"].data_ptr(),
                         a["n_free"].data_ptr(), 5, 1)


USUAL = [(B.uad_kv_attend_rows, rows_call()), (B.uad_kv_attend_rows, rows_call(row_start=None, q=rows_call()["q"][:3], out=rows_call()["q"][:3])),
         (B.uad_kv_attend_rows, rows_call(positions=ints(5), causal=False)), (B.uad_kv_reserve, reserve_call()),
         (B.uad_kv_reserve, reserve_call(new_tokens=None, row_start=None, slots=None)), (B.uad_kv_release, release_call())]


@pytest.mark.parametrize("call,args", USUAL)
def test_the_checks_in_c_hand_over_what_those_in_python_do(calls, monkeypatch, call, args):
    name = {B.uad_kv_attend_rows: "rows", B.uad_kv_reserve: "reserve", B.uad_kv_release: "release"}[call]
    used = []
    fast = getattr(B._marshal, name)
    monkeypatch.setattr(B._marshal, name, lambda *a: used.append(fast(*a)) or used[-1])
    call(**args)
    assert used == [0] and len(calls) == 1  # in C
    monkeypatch.setattr(B, "_marshal", None)
    call(**args)
    assert len(calls) == 2 and calls[0] == calls[1]


def test_the_checks_in_c_leave_odd_arguments_to_those_in_python(calls):
    B.uad_kv_attend_rows(**rows_call(scale=1))
    B.uad_kv_attend_rows(**rows_call(causal=1))
    B.uad_kv_attend_rows(**rows_call(kv=None))
    B.uad_kv_release(**release_call(kv=None))
    assert len(calls) == 4 and calls[1][-1] == 1 and calls[2][1] is None
    for f, n in ((B._marshal.rows, 16), (B._marshal.reserve, 13), (B._marshal.release, 10)):
        for bad in ((), (1,), (None,) * n, (1, "x") + (None,) * (n - 2)):
            assert f(*bad) is None
    a = release_call()
    order = [a[k] for k in ("kv", "lens", "page_table", "free_pages", "n_free", "window", "n_sinks", "n_pages", "device")]
    for i, odd in ((5, 2 ** 31), (5, 1.0), (6, None), (7, 8), (8, 0)):
        args = list(order)
        args[i] = odd
        assert B._marshal.release(B._release_at, *args) is None
    assert len(calls) == 4


def test_the_checks_in_c_keep_no_reference(calls):
    import sys
    a, b = rows_call(), reserve_call()
    tensors = [t for x in (a, b) for t in x.values() if isinstance(t, torch.Tensor)]
    before = [sys.getrefcount(t) for t in tensors]
    for _ in range(500):
        B.uad_kv_attend_rows(**a)
        B.uad_kv_reserve(**b)
        calls.clear()
    assert all(abs(x - sys.getrefcount(t)) < 20 for x, t in zip(before, tensors))


X5 = torch.zeros((5, HQ, HD))


REFUSED = ([(B.uad_kv_attend_rows, rows_call(**c)) for c in (
    dict(q=X5), dict(out=X5), dict(q=X5.half(), out=X5.half()), dict(q=X5[:, :2], out=X5[:, :2]), dict(q=X5[:4].bfloat16()), dict(q=None), dict(lens=None),
    dict(lens=ints(2)), dict(page_table=ints(3)), dict(row_start=ints(3)), dict(row_start=torch.zeros(4)), dict(positions=ints(3)), dict(device=0))]
    + [(B.uad_kv_reserve, reserve_call(**c)) for c in (
        dict(lens=ints(2)), dict(new_tokens=ints(4)), dict(free_pages=ints(8)), dict(n_free=ints(2)), dict(n_free_out=torch.zeros(1)), dict(n_free=3),
        dict(lens_out=ints(3).long()), dict(slots=ints(6)), dict(slots=torch.zeros((2, 3), dtype=torch.int64)), dict(row_start=ints(3)), dict(device=0),
        dict(slots=torch.zeros(12, dtype=torch.int64)[::2]), dict(page_table=ints(7, 3).t()))]
    + [(B.uad_kv_release, release_call(**c)) for c in (dict(lens=ints(2)), dict(free_pages=ints(10)), dict(n_free=None), dict(page_table=ints(3, 7).long()))])


@pytest.mark.parametrize("in_c", [True, False])
@pytest.mark.parametrize("call,change", REFUSED)
def test_the_binding_refuses_before_the_library(calls, monkeypatch, call, change, in_c):
    if not in_c:
        monkeypatch.setattr(B, "_marshal", None)
    with pytest.raises(ValueError):
        call(**change)
    assert not calls


def test_a_cache_with_block_scales_is_checked_before_the_library():
    for kw in (dict(block_scales=True), dict(block_scales=True, dtype=torch.float8_e4m3fn, k_scale=2.0), dict(k_scales=torch.zeros(1)),
               dict(v_scales=torch.zeros(1), dtype=torch.float8_e4m3fn)):
        with pytest.raises(ValueError):
            U.PagedKV(1, 1, 1, 64, 16, 4, 1, **kw)
