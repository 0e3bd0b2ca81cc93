"""Whole numbers of the paged cache's calls that 32 bits do not hold, in the binding, on CPU tensors (device -1): ctypes would
cut them to 32 bits, so that a window of 2^32 + 5 tokens became one of 5."""
import pytest
import torch

from tests.test_paged_rows_host import B, DEV, HD, HQ, calls, ints, release_call, reserve_call, rows_call  # noqa: F401

X = torch.zeros((3, HQ, HD), dtype=torch.bfloat16)
APPEND = dict(kv=0x1234, layer=2, k=X, v=X, page_table=ints(3, 7), lens=ints(3), row_start=None, positions=None, row_shape=(HQ, HD), device=DEV)
ATTEND = dict(kv=0x1234, layer=2, q=X, out=X, page_table=ints(3, 7), lens=ints(3), positions=None, scale=1.0, row_shape=(HQ, HD), device=DEV)
CREATE = dict(n_layers=1, n_heads=1, n_kv_heads=1, head_dim=64, page_size=16, n_pages=2, max_seqs=1, dtype=1, rope_dim=0, rope_pairs=0, rope_theta=1e4,
              k_scale=1.0, v_scale=1.0, k=X, v=X, stream=0)
PREFIX = dict(ctx=0x1234, kv=0x1234, lens=ints(3), page_table=ints(3, 7), prefix_len=8, device=DEV)


class NoCalls:
    """A library none of whose entry points is to be called."""

    def __getattr__(self, name):
        return lambda *a: pytest.fail(f"{name}{a}")


FAR = [2 ** 32, 2 ** 32 + 5, 2 ** 31, -2 ** 31 - 1, 2 ** 80, 5.0, "5", None]


@pytest.mark.parametrize("value", FAR)
@pytest.mark.parametrize("call,args,name", [
    (B.uad_kv_attend_rows, rows_call(), "window"), (B.uad_kv_attend_rows, rows_call(), "n_sinks"), (B.uad_kv_attend_rows, rows_call(), "layer"),
    (B.uad_kv_release, release_call(), "window"), (B.uad_kv_release, release_call(), "n_sinks"), (B.uad_kv_append, APPEND, "layer"),
    (B.uad_kv_attend, ATTEND, "layer"), (B.uad_set_prefix_paged, PREFIX, "prefix_len")] + [(B.uad_kv_create, CREATE, n) for n in list(CREATE)[:10]])
@pytest.mark.parametrize("in_c", [True, False])
def test_numbers_beyond_32_bits_are_refused(calls, monkeypatch, call, args, name, value, in_c):  # noqa: F811
    if not in_c:
        monkeypatch.setattr(B, "_marshal", None)
    monkeypatch.setattr(B, "load_library", NoCalls)
    with pytest.raises(ValueError, match=name):
        call(**{**args, name: value})
    assert not calls


class Long(torch.Tensor):
    """A tensor that says it is longer than it is."""
    n = 0

    @property
    def shape(self):
        return torch.Size((self.n,))


def test_more_slots_than_32_bits_count_are_refused(calls):  # noqa: F811
    slots = torch.zeros(6, dtype=torch.int64).as_subclass(Long)
    slots.n = 2 ** 32 + 6
    with pytest.raises(ValueError, match="slots"):
        B.uad_kv_reserve(**reserve_call(slots=slots))
    assert not calls


def test_numbers_of_32_bits_go_through(calls):  # noqa: F811
    B.uad_kv_attend_rows(**rows_call(window=2 ** 31 - 1, n_sinks=2 ** 31 - 1))
    assert calls[-1][-3:] == (2 ** 31 - 1, 2 ** 31 - 1, 1)
    B.uad_kv_release(**release_call(window=2 ** 31 - 1, n_sinks=-2 ** 31))
    assert calls[-1][-2:] == (2 ** 31 - 1, -2 ** 31)
