"""Status words of the cache and of an expert that reads it, against a stand-in for the HIP runtime."""
import ctypes

from tests.test_paged_host import OK, PAGE, ctx, kv, lib  # noqa: F401


def test_an_experts_status_is_cleared_before_synchronize_returns(lib, ctx):  # noqa: F811
    """On the context's stream: a clear that nothing waits for could take a following call's report with it."""
    lib.stub_log.restype = ctypes.c_char_p
    lib.stub_reset(-1)
    lib.kv_stub_ctx_status(ctx, 4)
    assert lib.uad_synchronize(ctx) == PAGE
    assert lib.stub_log() == b"sync copy sync "
    lib.stub_reset(-1)
    assert lib.uad_synchronize(ctx) == OK and lib.stub_log() == b"sync "


def test_a_caches_status_is_cleared_before_synchronize_returns(lib, kv):  # noqa: F811
    """Graphs of the handle's work may be replayed on other streams, which its own stream's clear is not ordered against."""
    lib.stub_log.restype = ctypes.c_char_p
    lib.stub_reset(-1)
    lib.kv_stub_status(kv, 4)
    assert lib.uad_kv_synchronize(kv) == PAGE and lib.stub_log() == b"sync sync "
    lib.stub_reset(-1)
    assert lib.uad_kv_synchronize(kv) == OK and lib.stub_log() == b"sync "
