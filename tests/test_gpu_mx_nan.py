"""NaN and infinities in what the attention over a cache in a microscaling format reads, at every number of query tiles and in both
formats: what they reach becomes NaN, everything else keeps its bits."""
import pytest
import torch

import mx_device as dev
from helpers import visible_new_keys
from paper_2402_11131_amd import api

pytestmark = pytest.mark.gpu
FP8, FP4 = api.SS_KV_MXFP8, api.SS_KV_MXFP4
ROWS = [(2, 1), (6, 1), (8, 2), (6, 4), (8, 4), (12, 3), (12, 4)]     # times two heads per KV head: one, two, .. five, six and eight tiles


def _problem(T, gamma, D, fmt):
    return dev.problem(11 * T + gamma, 1, T, gamma, 4, 2, D, 16, (600,), fmt, 600)


@pytest.mark.parametrize("T,gamma", ROWS)
@pytest.mark.parametrize("D,fmt", [(64, FP8), (128, FP8), (64, FP4), (128, FP4)])
def test_queries(T, gamma, D, fmt):
    d = _problem(T, gamma, D, fmt)
    clean = dev.call(d, gamma, 0.1)
    q = d["q"].clone()
    R = q.shape[1]
    bad = torch.zeros(R, 4, dtype=torch.bool, device=q.device)
    for r, h, i, v in ((0, 0, 3, float("inf")), (R - 1, 3, D - 1, float("nan")), (R // 2, 1, 40, float("-inf")), (R // 2, 2, 0, float("nan"))):
        q[0, r, h, i] = v
        bad[r, h] = True
    got = dev.call(dict(d, q=q), gamma, 0.1)
    assert torch.isfinite(clean).all() and torch.isnan(got[0][bad]).all() and torch.equal(got[0][~bad], clean[0][~bad])


@pytest.mark.parametrize("T,gamma", ROWS)
@pytest.mark.parametrize("D,fmt", [(64, FP8), (128, FP8), (64, FP4), (128, FP4)])
def test_cached_keys_and_values(T, gamma, D, fmt):
    d = _problem(T, gamma, D, fmt)
    clean = dev.call(d, gamma, 0.1)
    for pos in (0, 327, 599):
        page, slot = int(d["table"][0, pos // 16]), pos % 16
        for block in range(D // 32):
            c = [x.clone() for x in d["cache"]]
            c[1][page, 0, slot, block] = 255                   # a block of a key: every row of its KV head's two heads
            got = dev.call(dict(d, cache=c), gamma, 0.1)
            assert torch.isnan(got[0, :, :2]).all() and torch.equal(got[0, :, 2:], clean[0, :, 2:])
            c = [x.clone() for x in d["cache"]]
            c[3][page, 1, slot, block] = 255                   # of a value: its 32 features
            got = dev.call(dict(d, cache=c), gamma, 0.1)
            hit = torch.zeros(D, dtype=torch.bool, device=got.device)
            hit[32 * block:32 * block + 32] = True
            assert torch.isnan(got[0, :, 2:, hit]).all() and torch.equal(got[0, :, 2:, ~hit], clean[0, :, 2:, ~hit])
            assert torch.equal(got[0, :, :2], clean[0, :, :2])
        if fmt == FP8:
            c = [x.clone() for x in d["cache"]]
            c[0][page, 1, slot, D - 3] = 0xff                  # single elements may be NaN too
            c[2][page, 0, slot, 35] = 0x7f
            got = dev.call(dict(d, cache=c), gamma, 0.1)
            hit = torch.zeros(D, dtype=torch.bool, device=got.device)
            hit[35] = True
            assert torch.isnan(got[0, :, 2:]).all() and torch.isnan(got[0, :, :2, hit]).all()
            assert torch.equal(got[0, :, :2, ~hit], clean[0, :, :2, ~hit])


@pytest.mark.parametrize("T,gamma", ROWS)
@pytest.mark.parametrize("D,fmt", [(64, FP4), (128, FP8)])
def test_keys_of_the_step(T, gamma, D, fmt):
    """A NaN in a key reaches the rows that see it, and no other."""
    d = _problem(T, gamma, D, fmt)
    clean = dev.call(d, gamma, 0.1)
    sees = visible_new_keys(d["parent"][0].tolist(), gamma, False)
    R = T * (1 + gamma)
    for col in (T - 1, T, R - 1):
        k = d["k_new"].clone()
        k[0, col, 1, 7] = float("nan")
        got = dev.call(dict(d, k_new=k), gamma, 0.1)
        hit = torch.tensor([col in s for s in sees], device=got.device)
        assert hit.any() and torch.isnan(got[0, hit, 2:]).all()
        assert torch.equal(got[0, ~hit], clean[0, ~hit]) and torch.equal(got[0, :, :2], clean[0, :, :2])


@pytest.mark.parametrize("T,gamma", ROWS)
@pytest.mark.parametrize("D,fmt", [(64, FP8), (64, FP4), (128, FP8), (128, FP4)])
def test_what_lies_behind_a_sequence(T, gamma, D, fmt):
    """NaN scales and codes behind the last token change no bits, wherever in a block of 32 the sequence ends."""
    for L in (1, 15, 33, 511, 590):
        d = _problem(T, gamma, D, fmt)
        d["lens"].fill_(L)
        clean = dev.call(d, gamma, 0.1)
        c = [x.clone() for x in d["cache"]]
        page, slot = int(d["table"][0, (L - 1) // 16]), (L - 1) % 16 + 1
        keep = d["table"][0, :(L + 15) // 16].long()
        for x, y in zip(c, d["cache"]):
            x.fill_(255)
            x[keep] = y[keep]
            x[page, :, slot:] = 255
        assert torch.isfinite(clean).all() and torch.equal(dev.call(dict(d, cache=c), gamma, 0.1), clean), L
