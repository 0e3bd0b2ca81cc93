"""Appends whose sequences could touch more tiles in all than 32 bits count, which starts that fall make possible where the
page table is huge: refused by the host, as the plan on the device sums them up in 32 bits."""
import ctypes

import pytest

from tests.test_paged_host import ELEMS, OK, SHAPE, Pools, append, config, create, lib  # noqa: F401


@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_sums_of_tiles_fit_32_bits(lib, page):  # noqa: F811
    pools = Pools(lib, ELEMS * page // 16)
    st, h = create(lib, config(pools, page_size=page, max_seqs=2 ** 20))
    assert st == OK
    lib.kv_stub_reset(0)
    tile, most = min(page, 64), 2 ** 31 - 1
    for n_seqs in (2 ** 20, 2 ** 13, 1000, 65, 3):
        # the most tokens of a sequence whose tiles, and two that hold less, stay within 32 bits
        tokens = min((most // n_seqs - 2) * tile + tile - 1, 2 ** 31 - 2)
        # a call of as many rows, with page tables that do not matter, and one with page tables of as many tokens
        wide = 2 ** 30 // page
        if tokens < 2 ** 30:
            assert append(lib, h, n_rows=tokens, n_seqs=n_seqs, pages=wide) == OK
            assert append(lib, h, n_rows=tokens + 1, n_seqs=n_seqs, pages=wide) == SHAPE
            assert b"uad_kv_append: " in lib.uad_kv_last_error(h)
            pages = tokens // page
            assert append(lib, h, n_rows=most, n_seqs=n_seqs, pages=pages) == OK
            assert append(lib, h, n_rows=most, n_seqs=n_seqs, pages=pages + 1) == SHAPE
        else:
            assert append(lib, h, n_rows=most, n_seqs=n_seqs, pages=wide) == OK
    # a row per sequence: nothing to sum up
    assert append(lib, h, n_rows=2 ** 20, n_seqs=2 ** 20, pages=2 ** 30 // page, row_start=None) == OK
    lib.uad_kv_destroy(h)
    pools.close()


def test_the_bound_is_what_a_sequence_touches(lib):  # noqa: F811
    """Tokens within tiles of 16: a run of them touches two more tiles at most than it fills."""
    for n in range(0, 200):
        worst = max(((at + n - 1) // 16 - at // 16 + 1 if n else 0) for at in range(16))
        assert worst <= n // 16 + 2
