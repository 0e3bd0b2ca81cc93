"""The argument checks of the paged calls, in C for the usual case and in Python for every other: both hand the same to
the library, and what they refuse never gets there.  On CPU tensors (device -1), against a stand-in for the library."""
import ctypes

import pytest
import torch

import paper_2609_37772_amd as U

B = U._binding
HKV, HQ, HD, DEV = 2, 4, 64, -1
INTS = torch.int32
APPEND = ctypes.CFUNCTYPE(ctypes.c_int32, *U.load_library().uad_kv_append.argtypes)
ATTEND = ctypes.CFUNCTYPE(ctypes.c_int32, *U.load_library().uad_kv_attend.argtypes)


@pytest.fixture
def calls(monkeypatch):
    seen = []
    fns = [t(lambda *a: seen.append(a) or 0) for t in (APPEND, ATTEND)]
    monkeypatch.setattr(B, "_append_at", ctypes.cast(fns[0], ctypes.c_void_p).value)
    monkeypatch.setattr(B, "_attend_at", ctypes.cast(fns[1], ctypes.c_void_p).value)
    lib = type("Lib", (), {"uad_kv_append": staticmethod(fns[0]), "uad_kv_attend": staticmethod(fns[1]),
                           "uad_kv_last_error": staticmethod(lambda kv: b"")})
    monkeypatch.setattr(B, "load_library", lambda: lib)
    return seen


def rows(n, heads=HKV, dtype=torch.bfloat16):
    return torch.zeros((n, heads, HD), dtype=dtype)


def appended(n=5, seqs=3, **kw):
    a = dict(kv=0x1234, layer=2, k=rows(n), v=rows(n), page_table=torch.zeros((seqs, 7), dtype=INTS), lens=torch.zeros(seqs, dtype=INTS),
             row_start=torch.zeros(seqs + 1, dtype=INTS), positions=None, row_shape=(HKV, HD), device=DEV)
    a.update(kw)
    return a


def attended(seqs=3, **kw):
    a = dict(kv=0x1234, layer=0, q=rows(seqs, HQ), out=rows(seqs, HQ), page_table=torch.zeros((seqs, 7), dtype=INTS),
             lens=torch.zeros(seqs, dtype=INTS), positions=None, scale=0.125, row_shape=(HQ, HD), device=DEV)
    a.update(kw)
    return a


USUAL = [appended(), appended(row_start=None, n=3), appended(positions=torch.zeros(5, dtype=INTS)), appended(n=0), appended(n=1, seqs=1),
         appended(k=rows(5, dtype=torch.float32), v=rows(5, dtype=torch.float32))]
USUAL_ATTEND = [attended(), attended(seqs=1), attended(positions=torch.ones(3, dtype=INTS)),
                attended(q=rows(3, HQ, torch.float32), out=rows(3, HQ, torch.float32), scale=-2.5)]


@pytest.mark.parametrize("i", range(len(USUAL)))
def test_append_in_c_hands_over_what_python_does(calls, i):
    a = USUAL[i]
    checks = [a[k] for k in ("kv", "layer", "k", "v", "page_table", "lens", "row_start", "positions")]
    assert B._marshal.append(B._append_at, *checks, HKV, HD, DEV) == 0 and len(calls) == 1
    B._append_checked(*checks, (HKV, HD), DEV)
    assert calls[0] == calls[1] and calls[0][0] == 0x1234
    B.uad_kv_append(**a)
    assert calls[2] == calls[0]


@pytest.mark.parametrize("i", range(len(USUAL_ATTEND)))
def test_attend_in_c_hands_over_what_python_does(calls, i):
    a = USUAL_ATTEND[i]
    checks = [a[k] for k in ("kv", "layer", "q", "out", "page_table", "lens", "positions", "scale")]
    assert B._marshal.attend(B._attend_at, *checks, HQ, HD, DEV) == 0 and len(calls) == 1
    B._attend_checked(*checks, (HQ, HD), DEV)
    assert calls[0] == calls[1]
    B.uad_kv_attend(**a)
    assert calls[2] == calls[0]


WIDE = torch.zeros((5, 3 * HKV, HD), dtype=torch.bfloat16)


def test_slices_go_the_long_way_with_their_strides(calls):
    part = WIDE[:, HKV:2 * HKV]
    assert B._marshal.append(B._append_at, 1, 0, part, part, *[appended()[k] for k in ("page_table", "lens", "row_start", "positions")],
                             HKV, HD, DEV) is None
    B.uad_kv_append(**appended(k=part, v=rows(5)))
    assert len(calls) == 1 and calls[0][5:8] == (3 * HKV * HD, HKV * HD, 5)
    B.uad_kv_append(**appended(n=1, seqs=1, k=WIDE[:1, HKV:2 * HKV], v=rows(1)))
    assert calls[1][5:8] == (HKV * HD, HKV * HD, 1)


class Sub(torch.Tensor):
    pass


REFUSED = [
    dict(k=rows(5).half(), v=rows(5).half()), dict(k=rows(5).float()), dict(v=rows(4)), dict(k=rows(5, 3), v=rows(5, 3)),
    dict(k=rows(5)[:, :, :32], v=rows(5)[:, :, :32]), dict(k=rows(5).transpose(1, 2)), dict(k=rows(1).expand(5, HKV, HD)),
    dict(k=None), dict(v=[1]), dict(k=torch.zeros(5, HKV * HD, dtype=torch.bfloat16)), dict(page_table=torch.zeros((3, 7), dtype=torch.int64)),
    dict(page_table=torch.zeros(3, dtype=INTS)), dict(page_table=torch.zeros((7, 3), dtype=INTS).t()), dict(page_table=None),
    dict(lens=None), dict(lens=torch.zeros(2, dtype=INTS)), dict(lens=torch.zeros(3)), dict(lens=torch.zeros(6, dtype=INTS)[::2]),
    dict(row_start=torch.zeros(3, dtype=INTS)), dict(positions=torch.zeros(4, dtype=INTS)), dict(device=0)]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_append_refuses_before_the_library(calls, i):
    with pytest.raises(ValueError):
        B.uad_kv_append(**appended(**REFUSED[i]))
    assert not calls


@pytest.mark.parametrize("change", [dict(q=rows(2, HQ)), dict(out=rows(2, HQ)), dict(q=rows(2, HQ), out=rows(2, HQ)), dict(out=rows(3, HQ).float()),
                                    dict(q=rows(3), out=rows(3)), dict(positions=torch.zeros(2, dtype=INTS)), dict(device=1), dict(out=None)])
def test_attend_refuses_before_the_library(calls, change):
    with pytest.raises(ValueError):
        B.uad_kv_attend(**attended(**change))
    assert not calls


def test_unusual_but_good_arguments(calls):
    """Subclasses of a tensor, a whole number as the scale, a handle that was closed: the long way decides."""
    B.uad_kv_append(**appended(k=rows(5).as_subclass(Sub)))
    B.uad_kv_attend(**attended(scale=1))
    B.uad_kv_append(**appended(kv=None))
    assert len(calls) == 3 and calls[1][-1] == 1.0 and calls[2][0] is None
    for bad in ((), (1, 2), (None,) * 12, (B._append_at, "x", 0) + (None,) * 9, (B._append_at, 1, 2 ** 40) + (None,) * 9):
        assert B._marshal.append(*bad) is None and B._marshal.attend(*bad) is None
    assert len(calls) == 3


def test_no_reference_is_kept(calls):
    import sys
    a = appended()
    tensors = [a["k"], a["v"], a["page_table"], a["lens"], a["row_start"]]
    before = [sys.getrefcount(t) for t in tensors] + [sys.getrefcount(o) for o in (torch.bfloat16, INTS, torch.Tensor)]
    for _ in range(1000):
        B.uad_kv_append(**a)
        calls.clear()
        B._marshal.append(B._append_at, 1, 0, a["k"], None, a["page_table"], a["lens"], None, None, HKV, HD, DEV)
    after = [sys.getrefcount(t) for t in tensors] + [sys.getrefcount(o) for o in (torch.bfloat16, INTS, torch.Tensor)]
    assert all(abs(x - y) < 20 for x, y in zip(before, after))
