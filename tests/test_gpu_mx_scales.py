"""Attention over a cache in a microscaling format with scales at the ends of what is allowed."""
import ctypes

import numpy as np
import pytest
import torch

import mx_reference as ref
from helpers import to_np_f32
from paper_2402_11131_amd import api

DEV = "cuda:0"
FP8, FP4 = api.SS_KV_MXFP8, api.SS_KV_MXFP4


def _call(d, gamma, scale):
    return to_np_f32(api.ss_msa_attention_mx(d["q"], d["k_new"], d["v_new"], *d["cache"], d["table"], d["lens"], d["parent"], gamma, scale))


def _check(host, d, fmt, gamma, scale, page, L):
    K, V = ref.rows_of_cache(host["cache"], fmt, host["table"][0], L, page)
    want, tol = ref.attention(to_np_f32(host["q"][0]), to_np_f32(host["k_new"][0]), to_np_f32(host["v_new"][0]), K, V, host["parent"][0], gamma,
                              scale)
    off = np.abs(_call(d, gamma, scale)[0] - want)
    assert np.all(off <= tol), (off / tol).max()


@pytest.mark.gpu
@pytest.mark.parametrize("up", [10, 30, 60, 110])
@pytest.mark.parametrize("T,gamma,D,fmt", [(8, 2, 64, FP4), (40, 0, 64, FP4), (16, 4, 128, FP8), (33, 2, 128, FP4)])
def test_small_queries_and_a_large_scale(T, gamma, D, fmt, up):
    """Queries of 2^-up and a scale of 0.1 * 2^up: ordinary scores.  With more than 32 rows of the step's own there are rows that
    see none of a block of 32."""
    host, d = ref.problem(83, 1, T, gamma, 1, 1, D, 16, (64,), fmt)
    host["q"] *= 2.0 ** -up
    d["q"] = host["q"].to(DEV)
    _check(host, d, fmt, gamma, 0.1 * 2.0 ** up, 16, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("T,gamma", [(1, 0), (40, 0), (16, 4)])
@pytest.mark.parametrize("fmt", [FP8, FP4])
def test_scores_far_below_zero_before_a_small_scale(T, gamma, fmt):
    """Every score is -2^116, with the scale -128: all visible keys weigh the same."""
    D, page, L = 64, 16, 37
    host, d = ref.problem(87, 1, T, gamma, 2, 1, D, page, (L,), fmt)
    host["cache"][0][:] = 0xAA if fmt == FP4 else 0xB8     # -1 (e2m1: code 10, twice; e4m3: 0x38 with the sign)
    host["cache"][1][:] = 127 + 50
    host["q"][:] = 2.0 ** 60
    host["k_new"][:] = -2.0 ** 50
    for n in ("q", "k_new"):
        d[n] = host[n].to(DEV)
    d["cache"] = [torch.from_numpy(c).to(DEV) for c in host["cache"]]
    assert np.all(ref.rows_of_cache(host["cache"], fmt, host["table"][0], L, page)[0] == -2.0 ** 50)
    _check(host, d, fmt, gamma, 2.0 ** -109, page, L)


def test_a_scale_beyond_fp32_is_refused():
    P = ctypes.c_void_p(4096)   # never dereferenced
    call = lambda s: api.load_library().ss_msa_attention_mx(P, P, P, P, P, P, P, P, 8, 16, P, P, None, 1, 4, 2, 4, 2, 64, 16, ctypes.c_float(s), 1, 0, P, P,  # noqa: E731
                                                            0, None)
    for s in (2.5e38, 3.4e38, float("inf")):
        assert call(s) == 1 and b"scale" in api.load_library().ss_last_error()
