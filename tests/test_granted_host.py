"""Refusals of the calls that say, and go by, what sequences have room for. No call here reaches a kernel."""
import ctypes

from test_pages_host import INVALID, P, TOO_SMALL, b, h  # noqa: F401


def test_refusals(b, h):  # noqa: F811
    lib = b._lib
    q = b.us_kv_seqs(block_table=P, table_stride=10, lengths=P, cu_tokens=None, n_seqs=3, table_width=10)
    rows = (0, 256, 128, 256, 128)
    assert lib.us_kv_append_granted(h, ctypes.byref(q), 3, P, P, *rows, P + 2, None) == INVALID
    assert lib.us_kv_append_granted(None, ctypes.byref(q), 3, P, P, *rows, P, None) == INVALID
    assert lib.us_kv_append_granted(h, ctypes.byref(q), 3, None, P, *rows, P, None) == INVALID
    q.n_seqs = 0
    assert lib.us_kv_append_granted(h, ctypes.byref(q), 0, None, None, *rows, P, None) == 0
    extend = (P, P, 10, 10, P, 3, None, 1)
    assert lib.us_kv_extend_granted(h, *extend, P + 1, P, 1 << 30, None) == INVALID
    assert lib.us_kv_extend_granted(None, *extend, P, P, 1 << 30, None) == INVALID
    assert lib.us_kv_extend_granted(h, *extend, P, P, 100, None) == TOO_SMALL
    assert lib.us_kv_extend_granted(h, P, P, 10, 10, P, 0, None, 1, P, None, 0, None) == 0
