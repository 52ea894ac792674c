"""Attention over a cache in a microscaling format, splits so long that the waves load their page ids again: a wave (up to 32 query
rows per KV head) or a group of waves (more) holds those of 64 of its blocks of 32 tokens."""
import pytest
import torch
import torch

import mx_device as dev
from paper_2402_11131_amd import api

pytestmark = pytest.mark.gpu
FP8, FP4 = api.SS_KV_MXFP8, api.SS_KV_MXFP4
# T, gamma (query tiles), sequences (so that the plan has one split), tokens that 64 blocks of all waves or groups are
ROWS = [((1, 0), 48, 8192), ((4, 2), 48, 8192), ((6, 3), 16, 8192),            # one and two tiles: keys of a wave's own, four waves
        ((10, 3), 8, 8192), ((12, 4), 8, 6144), ((16, 4), 8, 6144),            # three, four, five: up to four, three, three groups
        ((24, 3), 16, 2048), ((24, 4), 16, 2048)]                              # six, eight: one group


@pytest.mark.parametrize("D,fmt,page", [(128, FP4, 16), (128, FP8, 64), (64, FP4, 64), (64, FP8, 16)])
@pytest.mark.parametrize("rows,B,reload", ROWS)
def test_page_ids_are_loaded_again(rows, B, reload, D, fmt, page):
    (T, gamma), Hkv, L = rows, 32, 17011
    assert api.ss_msa_mx_plan(B, T, gamma, Hkv, Hkv, D, L + page)[0] == 1 and L > 2 * reload
    # one sequence of two reloads and more, one of a bit more than one, the others short
    lens = [L, reload + 45] + [33 + b for b in range(B - 2)]
    d = dev.problem(200 + T + D, B, T, gamma, Hkv, Hkv, D, page, lens, fmt, L)
    out = dev.call(d, gamma, 0.05)
    for b, head in ((0, 0), (0, 17), (1, 31), (2, 3)):
        dev.check(d, out, fmt, gamma, 0.05, page, b, head)


@pytest.mark.parametrize("rows,B", [((1, 0), 16), ((16, 4), 4), ((24, 4), 8)])
def test_in_several_splits(rows, B):
    """The same with several long splits, of which the last is short."""
    (T, gamma), Hkv, D, page, L = rows, 8, 128, 64, 70001
    n, _ = api.ss_msa_mx_plan(B, T, gamma, Hkv, Hkv, D, L + page)
    assert n > 1 and L // n > (8192 if T == 1 else 4096)
    d = dev.problem(300 + T, B, T, gamma, Hkv, Hkv, D, page, [L] + [100] * (B - 1), FP4, L)
    out = dev.call(d, gamma, 0.05)
    for b, head in ((0, 0), (0, 7), (1, 3)):
        dev.check(d, out, FP4, gamma, 0.05, page, b, head)
    assert torch.equal(out, dev.call(d, gamma, 0.05))
