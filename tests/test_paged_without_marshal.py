"""The library without the argument checks in C: everything loads and runs, and the checks are made in Python."""
import importlib
import os
import subprocess
import sys

import pytest

from tests.test_paged_marshal import B, REFUSED, USUAL, USUAL_ATTEND, appended, calls  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def plain(calls, monkeypatch):  # noqa: F811
    monkeypatch.setattr(B, "_marshal", None)
    return calls


def test_the_library_loads_without_it():
    """In a process of its own, where the module cannot be imported."""
    code = ("import sys; sys.modules['paper_2609_37772_amd._marshal'] = None\n"
            "import paper_2609_37772_amd as U; U.load_library(); assert U._binding._marshal is None\n"
            "import numpy as np; print(U.uad_build_schedule(np.array([[1, 2]], np.int32))[0])")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "2", r.stderr


@pytest.mark.parametrize("call,args", [(B.uad_kv_append, a) for a in USUAL] + [(B.uad_kv_attend, a) for a in USUAL_ATTEND])
def test_calls_hand_over_the_same(calls, monkeypatch, call, args):  # noqa: F811
    call(**args)
    monkeypatch.setattr(B, "_marshal", None)
    call(**args)
    assert len(calls) == 2 and calls[0] == calls[1]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_append_refuses(plain, i):
    with pytest.raises(ValueError):
        B.uad_kv_append(**appended(**REFUSED[i]))
    assert not plain


def test_build_leaves_it_out_where_it_cannot_be_compiled(tmp_path, monkeypatch, capsys):
    build = importlib.import_module("paper_2609_37772_amd.build")
    old = tmp_path / "_marshal.so"
    for cc in ("false", "/no/such/compiler"):
        old.write_bytes(b"of older sources")
        monkeypatch.setattr(build, "MARSHAL", str(old))
        monkeypatch.setenv("CC", cc)
        build._compile_marshal()
        assert not old.exists() and "left out" in capsys.readouterr().err
