"""Launches of 2^32 threads and more, which the runtime cannot make, are refused before anything is enqueued (no GPU needed)."""
import ctypes

from paper_2402_11131_amd import api

P, OUT = ctypes.c_void_p(4096), ctypes.c_void_p(1 << 30)   # never dereferenced
UNSUPPORTED = 2


def _refused(rc):
    assert rc == UNSUPPORTED and b"grid too large" in api.load_library().ss_last_error()


def test_rows_and_heads_of_one_call():
    lib = api.load_library()
    # 32 rows of heads of 128 per workgroup of 256 threads: 2^24 workgroups are 2^32 threads
    for S, Hkv, D in ((1 << 26, 8, 128), ((1 << 26) - 31, 8, 128), (1 << 24, 64, 64), (1 << 30, 65535, 64)):
        _refused(lib.ss_kv_append_mx(P, P, P, P, P, P, P, 8, 16, P, P, 1, S, Hkv, D, 16, 1, 1, OUT, None))
        _refused(lib.ss_kv_read_mx(P, P, P, P, P, 8, 16, None, P, 1, S, Hkv, D, 16, 1, 1, P, P, None))


def test_sequences_and_heads_of_an_attention_call():
    lib = api.load_library()
    # workgroups of 256 threads; with 33 rows and more of up to 960 (T = 64 with 8 streams: several per sequence and head)
    for T, gamma, heads in ((1, 0, 257), (20, 1, 256), (64, 8, 64)):
        _refused(lib.ss_msa_attention_mx(P, P, P, P, P, P, P, P, 8, 16, P, P, None, 65535, T, gamma, heads, heads, 64, 16, ctypes.c_float(0.1), 1, 0,
                                         P, P, 1 << 40, None))
