"""Attention over caches in microscaling formats that are larger than 32-bit offsets reach, in both of its kernels: up to 32 query
rows per KV head (keys of a wave's own) and more (keys shared by waves)."""
import pytest
import torch

import mx_reference as ref
from helpers import to_np_f32
from paper_2402_11131_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FP8, FP4 = api.SS_KV_MXFP8, api.SS_KV_MXFP4


def _moved(d, pages):
    """The problem's cache at the end of a pool of `pages` pages, whose other pages hold whatever was there."""
    num = d["cache"][0].shape[0]
    cache = []
    for c in d["cache"]:
        big = torch.empty((pages,) + tuple(c.shape[1:]), dtype=torch.uint8, device=DEV)
        big[pages - num:] = c
        cache.append(big)
    return dict(d, cache=cache, table=d["table"] + (pages - num))


def _check(host, d, fmt, gamma, scale, page):
    out = to_np_f32(api.ss_msa_attention_mx(d["q"], d["k_new"], d["v_new"], *d["cache"], d["table"], d["lens"], d["parent"], gamma, scale))
    for b in range(out.shape[0]):
        K, V = ref.rows_of_cache(host["cache"], fmt, host["table"][b], int(host["lens"][b]), page)
        want, tol = ref.attention(to_np_f32(host["q"][b]), to_np_f32(host["k_new"][b]), to_np_f32(host["v_new"][b]), K, V, host["parent"][b],
                                  gamma, scale, device=DEV)
        assert abs(out[b] - want).max() < 1e3 and (abs(out[b] - want) <= tol).all(), b


# T, gamma with one query head per KV head or three: one tile; three, five tiles of a wave each; six and eight, two per wave
@pytest.mark.parametrize("T,gamma,heads", [(4, 1, 1), (16, 2, 1), (16, 4, 1), (30, 2, 1), (14, 2, 3)])
@pytest.mark.parametrize("fmt", [FP8, FP4])
def test_beyond_four_gib(T, gamma, heads, fmt):
    Hkv, D, page = 8, 128, 64
    host, d = ref.problem(71, 2, T, gamma, heads * Hkv, Hkv, D, page, (1000, 333), fmt)
    row = D if fmt == FP8 else D // 2
    _check(host, _moved(d, (1 << 32) // (row * page * Hkv) + 64), fmt, gamma, 0.1, page)


@pytest.mark.parametrize("T,gamma", [(4, 1), (16, 2), (16, 4), (30, 2)])
def test_beyond_two_to_the_31_rows(T, gamma):
    """Rows of 32 bytes, 2^31 of them: 64 GiB.  Keys and values, which are only read, are the same tensor."""
    Hkv, D, page = 8, 64, 64
    pages = (1 << 31) // (Hkv * page) + 64
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GiB of free device memory")
    host, d = ref.problem(73, 2, T, gamma, Hkv, Hkv, D, page, (700, 90), FP4)
    host["cache"][2:] = host["cache"][:2]
    num = d["cache"][0].shape[0]
    cache = []
    try:
        for c in d["cache"][:2]:
            cache.append(torch.empty((pages,) + tuple(c.shape[1:]), dtype=torch.uint8, device=DEV))
            cache[-1][pages - num:] = c
        _check(host, dict(d, cache=cache * 2, table=d["table"] + (pages - num)), FP4, gamma, 0.1, page)
    finally:
        cache.clear()
        torch.cuda.empty_cache()
