"""Where magnitudes held in a microscaling format end: what is rounded up to 2^128 reads as infinity, what lies below does not."""
import numpy as np
import pytest
import torch

import oracle
from paper_2402_11131_amd import api

FMTS = [api.SS_KV_MXFP8, api.SS_KV_MXFP4]
FIRST = {api.SS_KV_MXFP8: 1.9375, api.SS_KV_MXFP4: 1.75}   # times 2^127: half way to 2^128 from the element below it


def _rows(fmt):
    x = np.zeros((1, 4, 1, 64), np.float32)
    top = np.float32(2.0 ** 127)
    x[0, 0, 0, 3] = np.float32(FIRST[fmt]) * top
    x[0, 1, 0, 40] = -np.finfo(np.float32).max
    x[0, 2, 0, 5] = np.nextafter(np.float32(FIRST[fmt]), np.float32(0)) * top
    x[0, 3, 0, 63] = -top
    return x


def _check(got, fmt):
    below = {api.SS_KV_MXFP8: 1.875, api.SS_KV_MXFP4: 1.5}[fmt] * 2.0 ** 127
    assert got[0, 0, 0, 3] == np.inf and got[0, 1, 0, 40] == -np.inf
    assert got[0, 2, 0, 5] == below and got[0, 3, 0, 63] == -2.0 ** 127
    assert np.count_nonzero(got) == 4


@pytest.mark.parametrize("fmt", FMTS)
def test_oracle(fmt):
    with np.errstate(over="ignore"):
        _check(oracle.mx_values(*oracle.mx_quantise(_rows(fmt), fmt), fmt).astype(np.float32), fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", FMTS)
def test_append_and_read(fmt, out):
    dev = "cuda:0"
    cache = api.ss_kv_cache_mx(1, 1, 16, 64, fmt, dev)
    zero = torch.zeros(1, dtype=torch.int32, device=dev)
    rows = torch.from_numpy(_rows(fmt)).to(dev)
    new = api.ss_kv_append_mx(rows, rows, *cache, zero[None], zero, zero + 4)
    k, v = (torch.zeros((1, 4, 1, 64), dtype=out, device=dev) for _ in range(2))
    api.ss_kv_read_mx(*cache, zero[None], new, k, v)
    for x in (k, v):
        _check(x.float().cpu().numpy(), fmt)
