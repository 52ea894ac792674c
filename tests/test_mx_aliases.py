"""New lengths are written while other workgroups still read their inputs: calls on a cache in a microscaling format refuse an
output that shares memory with one (no GPU needed: nothing is enqueued)."""
import ctypes

import pytest

from paper_2402_11131_amd import api

INVALID = 1
B, COLS, DEPTH = 5, 8, 3
P = ctypes.c_void_p(1 << 20)   # never dereferenced
AT = dict(table=1 << 16, lens=2 << 16, count=3 << 16, path=4 << 16)
SIZE = dict(table=4 * B * COLS, lens=4 * B, count=4 * B, path=4 * B * (DEPTH + 1))


def _append(new):
    return api.load_library().ss_kv_append_mx(P, P, P, P, P, P, AT["table"], COLS, 16, AT["lens"], AT["count"], B, 4, 2, 64, 16, 1, 1, new, None)


def _commit(new):
    return api.load_library().ss_kv_commit_mx(P, P, P, P, P, P, AT["table"], COLS, 16, AT["lens"], AT["path"], AT["count"], B, 4, 2, 2, 64, 16, DEPTH, 1,
                                              1, new, None)


@pytest.mark.parametrize("call,names", [(_append, ("table", "lens", "count")), (_commit, ("table", "lens", "count", "path"))])
def test_new_lengths_share_no_memory_with_an_input(call, names):
    for name in names:
        for new in (AT[name], AT[name] + 4, AT[name] + SIZE[name] - 4, AT[name] - 4 * (B - 1)):
            assert call(new) == INVALID, (name, new - AT[name])
            assert b"shares memory" in api.load_library().ss_last_error()
